"""GPU tests of what a caller's own scales, lengths and windows may be in attention over 8-bit rows, and of how exact it is, against plain 64-bit implementations
(tests/quant_oracle.py)."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests import cache_oracle as O
from tests import quant_oracle as Q
from tests.test_gpu_cache import cache_of, near
from tests.test_gpu_quant import STORES, check, run_quant, run_tree, run_window, seed_of, trees_of

#: lens, new, room for more than 4096 tokens: tiles of 16, 32 (bf16), 128 and 256 rows (bf16), and split keys
SHAPES = {
    "few": ((90, 300, 64), (16, 4, 1), False),
    "drafts": ((90, 300), (7, 5), True),
    "rows": ((400, 700), (16, 20), True),
    "many_rows": ((400, 700), (100, 70), True),
    "split": ((6000,), (3,), False),
    "rows_split": ((6000,), (150,), False),
}


#: many rows of 128 at a time
CROWD = ((300,) * 48, (200,) * 48, True)


def setup(seed, store, dtype, shape, h=8, g=2, **more):
    lens, new, wide = SHAPES.get(shape, CROWD)
    return Q.QuantSetup(seed, store, dtype, h, g, 16, lens, new, spare_cols=256 if wide else 1, behind=1, **more)


def run_kind(st, kind, window=70, sinks=3):
    if kind == "quant":
        return run_quant(st, cache_of(st)), lambda b: Q.sees_range(st, b)
    if kind == "window":
        return run_window(st, cache_of(st), window, sinks), lambda b: Q.sees_window(st, b, window, sinks)
    mask = trees_of(st)
    return run_tree(st, cache_of(st), mask), lambda b: Q.sees_tree(st, b, mask)


# ---- signs ----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["quant", "window", "tree"])
@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("signs", ["all", "some", "large"])
def test_scales_below_zero(kind, store, dtype, shape, signs):
    """A caller's own scales: all below zero, of either sign, and those below zero 2^40 times as large as the others."""
    st = setup(seed_of(kind, store, dtype, shape, signs), store, dtype, shape, q_scale=2.0)
    for name in ("k_scales", "v_scales"):
        x = getattr(st, name)
        below = torch.rand(x.shape, generator=st.gen) < (1.0 if signs == "all" else 0.5 if signs == "some" else 0.1)
        x[below] *= -1.0
        if signs == "large" and name == "v_scales":
            x[below] *= 2.0 ** 40
    got, sees = run_kind(st, kind)
    check(st, got, sees, spread=signs == "large")


# ---- sizes ----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("power,others", [(120, 0.0), (120, 2.0 ** -100), (127, 0.0), (60, 2.0 ** -60)])
def test_the_sum_of_a_row_that_sees_a_far_larger_value(store, dtype, shape, power, others):
    """Some tokens' documents begin before a value of 2^power beside ones of 0 or next to it.  What makes most of every row's sum are many keys whose probabilities are
    2^-7 of the largest: none of them may be lost."""
    st = setup(seed_of(store, dtype, shape, power), store, dtype, shape)
    one, half = (127, 64) if store == "int8" else (1.0, 0.5)
    st.k_scales[:] = 1.0 / 127.0 if store == "int8" else 1.0
    st.q = torch.zeros_like(st.q)
    st.q[:, :, 0] = 110.0
    k = torch.zeros(st.k.shape)
    k[..., 0] = half
    st.v_scales[:] = others
    first = torch.randint(0, 2, (st.total,), generator=st.gen).int() * 8
    first[0], first[int(st.cu[-1]) - 1] = 0, 8
    for b in range(st.batch):
        k[int(st.table[b, 0]), :, 9:12, 0] = one                # the largest scores, seen by all
        st.v_scales[int(st.table[b, 0]), :, 5] = 2.0 ** power   # ... and seen from 0 on
    st.k = k.to(Q.CODES[store])
    st.v = (torch.randint(-1, 2, st.v.shape, generator=st.gen).float()).to(Q.CODES[store])
    got = run_quant(st, cache_of(st), first=first)
    check(st, got, lambda b: Q.sees_range(st, b, None, first), spread=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_scales_next_to_the_largest_number(dtype, shape):
    """Scales of 2^126 under codes of 2^-9 and none, in tiles of which a page is missing; scores that grow by less than 16 times, under a maximum that lags."""
    st = setup(seed_of(dtype, shape), "fp8", dtype, shape)
    st.k_scales[:] = 1.0
    st.q = torch.zeros_like(st.q)
    st.q[:, :, 0] = 31.0
    k = torch.zeros(st.k.shape)
    for b, s in enumerate(st.lens):
        for c in range(-(-s // 16)):
            k[int(st.table[b, c]), :, :, 0] = min(c // 4, 7) / 8     # (31 / sqrt(128) / 8 is half a power of two)
    st.k = k.to(Q.CODES["fp8"])
    st.v = (torch.randint(-1, 2, st.v.shape, generator=st.gen).float() * 2.0 ** -9).to(Q.CODES["fp8"])
    st.v_scales[:] = 2.0 ** 126
    for b, s in enumerate(st.lens):
        st.table[b, 1:-(-s // 16):2] = -1
    check(st, run_quant(st, cache_of(st)), lambda b: Q.sees_range(st, b), spread=True)


# ---- windows --------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("store", ["plain"] + STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [(1, 1), (40, 10), (300, 4)])
@pytest.mark.parametrize("cur,window", [(1 << 22, (1 << 22) - 100), (1 << 22, 1 << 22), (1 << 29, 2 ** 31 - 1), ((1 << 30) - 1, 1 << 30)])
def test_wide_windows_far_beyond_the_table(store, dtype, new, cur, window):
    """Tokens millions of slots beyond the table's, in windows that reach back into it."""
    st = Q.QuantSetup(seed_of(store, dtype, new, cur), store, dtype, 8, 2, 16, (320, 64), new, spare_cols=0)
    st.cur = torch.tensor([cur, cur - 30], dtype=torch.int32)
    got = run_window(st, cache_of(st), window, 3)

    def sees(b):
        last = int(st.cur[b])
        pos, t = torch.arange(last - new[b], last)[:, None], torch.arange(st.cols * 16)[None, :]
        return (t <= pos) & ((t > pos - window) | (t < 3))
    st.lens = [320, 320]
    check(st, got, sees)


# ---- weights --------------------------------------------------------------------------------------------------
def pairs(store, dtype, shape):
    """Keys of which two, of nearly the same score, have nearly all of a row's probability, and values of equal size and opposite sign: what is left of their difference is small
    beside what a rounding of either weight makes.  Queries have three elements, so that scores are nearly exact."""
    st = setup(seed_of(store, dtype, shape), store, dtype, shape, h=8, g=2)
    st.q = torch.zeros_like(st.q)
    st.q[:, :, 0] = 60.0
    st.q[:, :, 1:3] = 2.0 * torch.randn((st.total, 8, 2), generator=st.gen).to(st.td)
    one = 127.0 if store == "int8" else 448.0
    k = torch.zeros(st.k.shape)
    k[..., 0] = -one
    k[..., 1:3] = (torch.randn(k[..., 1:3].shape, generator=st.gen) * one / 8).clamp(-one, one)
    v = torch.randn(st.v.shape, generator=st.gen) * one / 8
    st.k_scales = (0.9 + 0.2 * torch.rand(st.k_scales.shape, generator=st.gen)) / one
    st.v_scales = (1.0 + torch.rand(st.v_scales.shape, generator=st.gen)) / one
    for b, s in enumerate(st.lens):
        at = (s - st.new[b]) // 2
        for i, sign in enumerate((1.0, -1.0)):
            page, row = int(st.table[b, (at + i) // 16]), (at + i) % 16
            k[page, :, row, 0] = one
            st.k_scales[page, :, row] = 1.0 / one
            v[page, :, row] = sign * torch.where(torch.arange(128) % 2 == 0, one, -one / 2)
            st.v_scales[page, :, row] = 1.37 / one
    st.k, st.v = ((x.round() if store == "int8" else x).to(Q.CODES[store]) for x in (k, v))
    return st


def weights_bound(st, sees, half):
    """Outputs, and how far off they may be if weights are off by `half` of themselves, scores by a step for each product, factor and sum, and sums by one for each key."""
    out, _, _, _ = Q.attention(st, sees)
    size, tol = torch.zeros_like(out), torch.zeros_like(out)
    G = st.h // st.g
    for b in range(st.batch):
        s, n, c0 = st.lens[b], st.new[b], int(st.cu[b])
        seen = sees(b)
        for kv in range(st.g):
            k, v = st.held("k", b, kv, s)[0], st.held("v", b, kv, s)[0]
            q = st.q[c0:c0 + n].to(O.F8).view(n, st.g, G, 128)[:, kv].transpose(0, 1)
            z = (torch.matmul(q, k.T) / math.sqrt(128.0)).masked_fill(~seen, -math.inf)
            err = float((torch.matmul(q.abs(), k.abs().T) / math.sqrt(128.0)).max()) * (8 if st.dtype == "bf16" else 16) * 2.0 ** -23 + 2.0 ** -20
            size = torch.matmul(torch.softmax(z, dim=-1), v.abs())
            rel = math.expm1(2 * err) + half + ((1 if st.dtype == "bf16" else 3) * s + 16) * 2.0 ** -23
            tol[c0:c0 + n, kv * G:(kv + 1) * G] = (size * rel).transpose(0, 1)
    return out, tol + out.abs() * O.HALF[st.dtype]


@pytest.mark.parametrize("kind", ["quant", "window", "tree"])
@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_weights_are_off_by_half_a_step_of_fp16(kind, store, dtype, shape):
    """... in bf16, by 2^-22 of themselves in fp32: not by the 2^-8 that bf16 weights would be off by, which the same bound refuses."""
    st = pairs(store, dtype, shape)
    got, sees = run_kind(st, kind, window=5000, sinks=0)
    want, tol = weights_bound(st, sees, 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22)
    near(got[0][:int(st.cu[-1])], want, tol, "out")


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [shape for shape in SHAPES if max(SHAPES[shape][1]) > 1])
@pytest.mark.parametrize("power", [20, 60, 120])
def test_weights_beside_large_values_are_as_exact(store, dtype, shape, power):
    """The last token of a sequence brings a value 2^power times as large as the others: those before it, which do not see it, are as exact as without."""
    st = pairs(store, dtype, shape)
    for b, (s, n) in enumerate(zip(st.lens, st.new)):
        if n > 1:
            st.v_scales[int(st.table[b, (s - 1) // 16]), :, (s - 1) % 16] *= 2.0 ** power
    out = run_quant(st, cache_of(st))[0][:int(st.cu[-1])].cpu()
    hit = [int(st.cu[b + 1]) - 1 for b, n in enumerate(st.new) if n > 1]
    assert torch.isfinite(out[hit]).all() and (out[hit].abs().amax(dim=-1) > 1e-7 * 2.0 ** power).all()     # (a hundred times e^-10 of it, at least, in some element)
    for b, (s, n) in enumerate(zip(st.lens, st.new)):
        if n > 1:
            st.v_scales[int(st.table[b, (s - 1) // 16]), :, (s - 1) % 16] *= 2.0 ** -power
    want, tol = weights_bound(st, lambda b: Q.sees_range(st, b), 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22)
    keep = torch.ones(len(out), dtype=torch.bool)
    keep[hit] = False
    near(out[keep], want[keep], tol[keep], "out")


@pytest.mark.parametrize("kind", ["quant", "window", "tree"])
@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weights_of_a_crowd(kind, store, dtype):
    """77 thousand rows: a weight in some ten thousand lies, rounded to fp32, half way between two numbers of fp16.  Its parts with fp32 queries have to be of one rounding."""
    st = pairs(store, dtype, "crowd")
    got, sees = run_kind(st, kind, window=5000, sinks=0)
    want, tol = weights_bound(st, sees, 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22)
    near(got[0][:int(st.cu[-1])], want, tol, "out")
