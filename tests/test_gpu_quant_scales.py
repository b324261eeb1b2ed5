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


def setup(seed, store, dtype, shape, h=8, g=2, **more):
    lens, new, wide = SHAPES[shape]
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
