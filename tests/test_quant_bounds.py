"""The bounds that tests/test_gpu_quant_scales.py holds weights over 8-bit rows to, on the CPU: weights of the types that the header names keep them, and coarser ones do not."""
import math

import pytest

torch = pytest.importorskip("torch")

from tests import cache_oracle as O
from tests import quant_oracle as Q
from tests import test_gpu_quant_scales as S


def outputs(st, weight):
    """Causal attention whose weights, probabilities times values' scales, are rounded to a type."""
    out = torch.zeros((int(st.cu[-1]), st.h, 128), dtype=O.F8)
    G = st.h // st.g
    for b in range(st.batch):
        s, n, c0, t = st.lens[b], st.new[b], int(st.cu[b]), torch.arange(st.lens[b])
        for kv in range(st.g):
            k, v = st.held("k", b, kv, s)[0], st.held("v", b, kv, s)[0]
            scale = st.v_scales[st.table[b, t // st.page].long(), kv, t % st.page].to(O.F8)
            q = st.q[c0:c0 + n].to(O.F8).view(n, st.g, G, 128)[:, kv].transpose(0, 1)
            z = (torch.matmul(q, k.T) / math.sqrt(128.0)).masked_fill(~Q.sees_range(st, b), -math.inf)
            p = torch.exp(z - z.amax(dim=-1, keepdim=True))
            o = torch.matmul((p * scale).to(weight).to(O.F8), v / scale[:, None]) / p.sum(dim=-1, keepdim=True)
            out[c0:c0 + n, kv * G:(kv + 1) * G] = o.transpose(0, 1)
    return out.to(st.td).to(O.F8)


@pytest.mark.parametrize("store", S.STORES)
@pytest.mark.parametrize("shape", ["few", "drafts", "rows", "many_rows"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_bounds_tell_weights_apart(store, shape, dtype):
    # (with fp32 queries sums of 700 keys may be off by 3 * 700 * 2^-23, half of what fp16 weights may be: there bf16 ones are refused)
    kept, refused = (torch.float16, torch.bfloat16) if dtype == "bf16" else (torch.float32, torch.float16 if max(S.SHAPES[shape][0]) <= 300 else torch.bfloat16)
    st = S.pairs(store, dtype, shape)
    want, tol = S.weights_bound(st, lambda b: Q.sees_range(st, b), 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22)
    assert ((outputs(st, kept) - want).abs() <= tol).all()
    assert ((outputs(st, refused) - want).abs() > tol).any(dim=-1).any(dim=-1).float().mean() > 0.5     # of the tokens
