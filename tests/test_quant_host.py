"""The operators on a paged KV cache of 8-bit rows, in windows and for drafted tokens without a GPU: refusals and devices, against the stand-in for the HIP
runtime (host_runtime/); what a token sees and which tiles a window goes through, in the kernels' own functions compiled for the host; the binding's checks; the
plain 64-bit quantisation that the GPU tests compare with."""
import os
import subprocess
import sys

import pytest

from tests.host_runtime.quant_scenarios import SCENARIOS

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
    r = subprocess.run([sys.executable, "-m", "tests.host_runtime.quant_scenarios", name, fake], cwd=ROOT, capture_output=True, text=True,
                       timeout=120)
    assert r.returncode == 0 and r.stdout.endswith("ok\n"), r.stdout + r.stderr


SIGHTS = r"""
#include "cache_args.hpp"
#include <cstdio>
#include <climits>
#include <initializer_list>
#include <vector>
using namespace ctkvr;
#define WANT(x) do { if (!(x)) { printf("failed: %s (%s:%d)\n", #x, __FILE__, __LINE__); return 1; } } while (0)
int main()
{
    const int odd[] = {INT32_MIN, -1, 0, 1, 31, 32, 33, 63, 64, 65, 100, 127, 200, INT32_MAX};
    for (int n : {-5, 0, 1, 31, 32, 40, INT_MIN, INT_MAX}) {
        const uint32_t w = low_bits(n);
        for (int i = 0; i < 32; ++i) WANT((w >> i & 1) == (i < n ? 1u : 0u));
    }
    // 128 slots; 40 new tokens, or lengths and token ranges that make no sense
    int32_t cu[2] = {0, 40}, cur[1] = {100};
    const int32_t table[8] = {0, 1, 2, 3, 4, 5, 6, 7};
    CacheView v{};
    v.table = table; v.cu = cu; v.cur = cur; v.batch = 1; v.h = 4; v.g = 2; v.lg = 1; v.page_shift = 4; v.max_pages = 8; v.total = 40; v.num_pages = 8;
    std::vector<int32_t> first(40);
    for (int words : {1, 2, 3}) {
        std::vector<uint32_t> mask(40 * words);   // (its end is the end of the allocation: a read beyond it is a sanitizer's matter, and is counted here by hand)
        uint32_t x = 1;
        for (auto &m : mask) m = x = x * 1664525u + 1013904223u;
        for (int c : odd) for (int e : odd) for (int f : {-3, 0, 50, 90, INT32_MAX}) {
            cur[0] = c; cu[1] = e;
            for (auto &y : first) y = f;
            const SeqSpan s = seq_span(v, 0);
            ScoreOpts o{};
            o.first = first.data(); o.drafts = mask.data(); o.words = words;
            for (int i = 0; i < s.n; i += 7) {
                const RowSight r = sight_of<kTree>(v, o, s, 0, i);
                for (int key0 = 0; key0 < 160; key0 += 32) {
                    const uint32_t w = sight_bits<kTree>(o, s, r, i, key0);
                    for (int k = 0; k < 32; ++k) {
                        const int64_t t = key0 + k, j = t - s.old;
                        bool sees = r.pos >= 0 && t < s.len && t >= (f > 0 ? f : 0);
                        if (j >= 0) sees = sees && j < 32 * words && (mask[(s.c0 + i) * words + j / 32] >> (j % 32) & 1);
                        WANT((bool)(w >> k & 1) == sees);
                    }
                }
            }
            o.first = nullptr;
            for (int window : {1, 5, 32, 1 << 21}) for (int sinks : {0, 1, 33, 64, 1 << 20}) {
                o.window = window; o.sinks = sinks;
                for (int i = 0; i < s.n; i += 7) {
                    const RowSight r = sight_of<kWindow>(v, o, s, 0, i);
                    WANT(r.lo >= 0 && r.hi >= 0 && r.hi <= s.len);
                    for (int key0 = 0; key0 < 160; key0 += 32) {
                        const uint32_t w = sight_bits<kWindow>(o, s, r, i, key0);
                        for (int k = 0; k < 32; ++k) {
                            const int64_t t = key0 + k;
                            WANT((bool)(w >> k & 1) == (t <= r.pos && t < s.len && (t > (int64_t)r.pos - window || t < sinks)));
                        }
                    }
                }
                // tiles: ascending, each once, inside the keys, and all that some token sees
                for (int keys : {32, 64}) {
                    if (!s.n) continue;
                    const RowSight a = sight_of<kWindow>(v, o, s, 0, 0), z = sight_of<kWindow>(v, o, s, 0, s.n - 1);
                    const KeyTiles kt = window_tiles(o, a.lo, z.hi, keys);
                    int before = -1;
                    bool there[5] = {};
                    for (int i = kt.from; i < kt.to; ++i) {
                        const int t = kt.at(i);
                        WANT(t > before && t * keys < z.hi);
                        there[t] = true;
                        before = t;
                    }
                    for (int t = 0; t < z.hi; ++t)
                        for (int i = 0; i < s.n; ++i) {
                            const RowSight r = sight_of<kWindow>(v, o, s, 0, i);
                            if (t < r.hi && (t >= r.lo || t < sinks)) WANT(there[t / keys]);
                        }
                    if (sinks == 0 && a.pos >= 0 && z.hi > a.lo) WANT(kt.to == (z.hi + keys - 1) / keys - a.lo / keys);
                }
            }
        }
    }
    // a row's sight by position is what it was
    cur[0] = 100; cu[1] = 40;
    const SeqSpan s = seq_span(v, 0);
    ScoreOpts o{};
    const RowSight r = sight_of<kRange>(v, o, s, 70, 3);
    WANT(r.lo == 0 && r.hi == 70 && r.pos == 63);
    WANT(sight_bits<kRange>(o, s, r, 3, 64) == 0x3fu && sight_bits<kRange>(o, s, r, 3, 32) == ~0u && sight_bits<kRange>(o, s, r, 3, 96) == 0);
    printf("ok\n");
}
"""


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="no hipcc")
def test_what_a_token_sees_and_the_tiles_of_a_window(tmp_path):
    src, exe = tmp_path / "host.hip", tmp_path / "host"
    src.write_text(SIGHTS)
    subprocess.run([HIPCC, "--offload-arch=gfx950", "--cuda-host-only", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2512_15550_amd", "csrc"),
                    "-o", str(exe), str(src)], check=True, capture_output=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout + r.stderr


def test_the_plain_quantisation():
    """Nearest codes, ties to even, in both kinds, against all of them."""
    import torch
    from tests import quant_oracle as Q
    x = torch.randn((40, 128), generator=torch.Generator().manual_seed(3))
    x[0] = 0.0
    x[1] = (torch.arange(128) - 64) / 4.0
    x[1, 0] = 63.5
    x[2, 5] = float("inf")
    x[3, 6] = float("nan")
    x[4] = torch.linspace(-448, 448, 128).round()
    x[5, 1:] *= 2.0 ** -14
    for store in ("int8", "fp8"):
        codes, scales, y = Q.quantised(x, store)
        every = torch.arange(-127, 128).double() if store == "int8" else torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().double()
        every = every[torch.isfinite(every)].unique()
        near = (y[..., None] - every).abs()
        assert ((y - codes).abs() == near.amin(dim=-1)).all()
        for value, code in ((64.5, 64.0), (-63.5, -64.0), (0.5, 0.0)) if store == "int8" else ((17.0, 16.0), (19.0, 20.0), (2.0 ** -10, 0.0)):
            row = torch.zeros(128)
            row[0], row[1] = Q.TOP[store], value
            assert Q.quantised(row[None], store)[0][0, 1] == code
        assert torch.isnan(scales[2]) and torch.isnan(scales[3]) and not codes[[0, 2, 3]].any() and scales[0] == 0


def test_the_binding_refuses_types_and_shapes():
    import types

    import torch

    import paper_2512_15550_amd as ck
    from paper_2512_15550_amd import _marshal
    from paper_2512_15550_amd import binding as B
    c = types.SimpleNamespace(torch_dtype=torch.bfloat16, _float=torch.float32, device=-1, _pointer=_marshal.pointer, _pointers=_marshal.pointers, _rows=_marshal.rows,
                              _formats={torch.bfloat16: ck.KV_PLAIN, torch.int8: ck.KV_INT8, torch.float8_e4m3fn: ck.KV_FP8},
                              _shapes={"pages": (3, 2, 16, 128), "scales": (3, 2, 16)})
    codes, scales = torch.zeros((3, 2, 16, 128), dtype=torch.int8), torch.zeros((3, 2, 16))
    assert B._format_of(c, codes) == ck.KV_INT8 and B._format_of(c, codes.view(torch.float8_e4m3fn)) == ck.KV_FP8
    plain = torch.zeros((3, 2, 16, 128), dtype=torch.bfloat16)
    assert B._format_of(c, plain, True) == ck.KV_PLAIN
    for x, ok in ((plain, False), (plain.float(), True), (codes.view(torch.uint8), True), (codes.view(torch.float8_e5m2), True)):
        with pytest.raises(ValueError):
            B._format_of(c, x, ok)
    assert B._all_on(c, *B._quant_of(c, codes, scales, codes, scales)) == (codes.data_ptr(), scales.data_ptr()) * 2
    assert B._all_on(c, *B._quant_of(c, None, None, codes, scales)) == (None, None, codes.data_ptr(), scales.data_ptr())
    for bad in ((codes, scales, codes.view(torch.float8_e4m3fn), scales), (codes, scales.double(), codes, scales), (codes, scales[:2], codes, scales),
                (codes[:, :, :, :64], scales, codes, scales), (codes, scales, codes.transpose(0, 1), scales)):
        with pytest.raises(ValueError, match="expected a contiguous"):
            B._all_on(c, *B._quant_of(c, *bad))


def test_tensors_are_checked_as_they_are_described():
    """The compiled checks against what torch says of the tensors: type, shape, order, device, strides of rows."""
    import torch

    from paper_2512_15550_amd import _marshal as M
    t = torch.zeros((6, 4, 16, 128), dtype=torch.bfloat16)
    assert M.pointer(t, torch.bfloat16, (6, 4, 16, 128), -1) == t.data_ptr() == M.pointer(t, torch.bfloat16, t.shape, -1)
    assert M.pointer(t[2:], torch.bfloat16, (4, 4, 16, 128), -1) == t[2:].data_ptr()
    one = t[:, :1].contiguous()
    assert M.pointer(one.transpose(0, 1), torch.bfloat16, (1, 6, 16, 128), -1) == one.data_ptr()      # (as contiguous as it was)
    for bad, dtype, shape, device in ((t, torch.float16, t.shape, -1), (t, torch.bfloat16, (6, 4, 16), -1), (t, torch.bfloat16, (6, 4, 16, 127), -1),
                                      (t, torch.bfloat16, (6, 4, 128, 16), -1), (t, torch.bfloat16, t.shape, 0), (t.transpose(0, 1), torch.bfloat16, (4, 6, 16, 128), -1),
                                      (t[:, ::2], torch.bfloat16, (6, 2, 16, 128), -1), ([1], torch.bfloat16, (1,), -1), (None, torch.bfloat16, (1,), -1),
                                      (t, "bf16", t.shape, -1), (t, torch.bfloat16, [6, 4, 16, 128], -1), (t.to_sparse(), torch.bfloat16, t.shape, -1)):
        assert M.pointer(bad, dtype, shape, device) == -1
        if bad is not None:
            assert M.pointers(device, "t", t, torch.bfloat16, t.shape, "none", None, 1, 2, "bad", bad, dtype, shape) == (2 if device == -1 else 0)
    assert M.pointer(t) == -1 and M.pointers(-1) == ()
    with pytest.raises(TypeError):
        M.pointers(-1, "t", t)
    empty = torch.zeros((0, 4), dtype=torch.int32)
    assert M.pointer(empty, torch.int32, (0, 4), -1) == empty.data_ptr()
    fused = torch.zeros((5, 12 * 128 + 64), dtype=torch.float32)
    q = fused[:, :1024].view(5, 8, 128)
    assert M.rows(q, torch.float32, 5, 8, -1) == (q.data_ptr(), 12 * 128 + 64)
    assert M.rows(q[:1], torch.float32, 1, 8, -1) == (q.data_ptr(), 1024)
    assert M.rows(q[:0], torch.float32, 0, 8, -1) == (q[:0].data_ptr(), 1024)
    assert M.rows(fused[:, 64:192].view(5, 1, 128), torch.float32, 5, 1, -1) == (fused[:, 64:].data_ptr(), 12 * 128 + 64)
    for bad in (q.bfloat16(), q[:4], q[:, :4], q[..., :64], q.flip(1)[:, :, ::2], q.transpose(1, 2), q[:, ::2], q.reshape(5, 1024), None, 7):
        assert M.rows(bad, torch.float32, 5, 8, -1) is None
