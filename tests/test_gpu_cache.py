"""GPU tests of the operators on the paged KV cache against plain 64-bit implementations (tests/cache_oracle.py): append, attention of new
tokens, accumulated weights, eviction, and a run of them together with the index."""
import math
import zlib

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2512_15550_amd as ck
from tests import cache_oracle as O

DEV = "cuda"
NAN = float("nan")


def cache_of(st, **over):
    p = dict(batch=st.batch, n_q_heads=st.h, n_kv_heads=st.g, num_pages=st.num_pages, max_pages=st.cols, max_new=max(st.total, 1),
             page_size=st.page, dtype=ck.BF16 if st.dtype == "bf16" else ck.F32)
    p.update(over)
    return ck.ctkvr_cache_create(ck.CacheParams(**p))


def near(got, want, tol, what):
    got, want = got.cpu().to(O.F8), want.to(O.F8)
    assert torch.equal(torch.isfinite(got), torch.isfinite(want)), f"{what}: finite values in other places"
    fin = torch.isfinite(want)
    assert torch.equal(got[~fin & ~torch.isnan(want)], want[~fin & ~torch.isnan(want)]), f"{what}: other infinities"
    off = (got - want).abs()[fin]
    over = off - tol[fin]
    assert not (over > 0).any(), f"{what}: off by {float(off[over.argmax()]):.3g} where {float(tol[fin][over.argmax()]):.3g} is allowed"


def dev(x):
    return None if x is None else x.to(DEV)


def run_attn(st, cache, q=None, **masks):
    out = torch.full((st.total, st.h, 128), 7.0, dtype=st.td, device=DEV)
    lse = torch.full((st.total, st.h), 7.0, device=DEV)
    ck.ctkvr_cache_attn(cache, dev(st.q) if q is None else q, dev(st.k), dev(st.v), dev(st.cu), dev(st.cur), dev(st.table), out, out_lse=lse,
                        slopes=dev(masks.get("slopes")), prefix_lens=dev(masks.get("prefix")), first_key=dev(masks.get("first")))
    torch.cuda.synchronize()
    return out, lse


def check_attn(st, cap=0.0, **masks):
    cache = cache_of(st, softcap=cap)
    out, lse = run_attn(st, cache, **masks)
    want, want_lse, tol, tol_lse = O.attention(st, cap=cap, **masks)
    n = int(st.cu[-1])
    near(out[:n], want, tol, "out")
    near(lse[:n], want_lse, tol_lse, "lse")
    assert (out[n:] == 7).all() and (lse[n:] == 7).all(), "tokens behind the last sequence were written"
    return cache, lse


def check_weights(st, cache, lse, cap=0.0, decay=1.0, with_in=True, **masks):
    width = st.cols * st.page + 3
    w_in = torch.rand((st.batch, st.g, width), generator=st.gen) if with_in else None
    w_out = torch.full((st.batch, st.g, width), 5.0, device=DEV)
    ck.ctkvr_cache_weights(cache, dev(st.q), lse, dev(st.k), dev(st.cu), dev(st.cur), dev(st.table), dev(w_in), w_out, decay=decay,
                           slopes=dev(masks.get("slopes")), prefix_lens=dev(masks.get("prefix")), first_key=dev(masks.get("first")))
    want, tol = O.weights(st, lse.cpu(), w_in, torch.full((st.batch, st.g, width), 5.0), decay, cap=cap, **masks)
    near(w_out, want, tol, "weights")
    return w_out


# lens, new: one token, tile edges of keys (32, 64) and rows, none at all, an empty cache
SHAPES = {
    "one": ((1,), (1,)),
    "single_tokens": ((64, 65, 1, 700), (1, 1, 1, 1)),
    "edges": ((31, 32, 33, 63, 64, 65), (31, 1, 33, 2, 64, 65)),
    "none": ((50, 0, 130), (0, 0, 130)),
    "chunk": ((300, 129), (128, 127)),
    "long_single": ((5000, 3), (1, 3)),
    "prompt": ((517,), (517,)),
}
HEADS = [(4, 4), (4, 2), (8, 2), (16, 2)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h,g", HEADS)
def test_attention_and_weights(shape, dtype, h, g):
    lens, new = SHAPES[shape]
    st = O.Setup(zlib.crc32(f"{shape} {dtype} {h}".encode()) % 1000, dtype, h, g, 16, lens, new, q_scale=2.0)
    cache, lse = check_attn(st)
    check_weights(st, cache, lse, decay=0.75)


@pytest.mark.parametrize("page", [1, 2, 32, 64, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_page_sizes(page, dtype):
    st = O.Setup(page, dtype, 8, 2, page, (page + 70, 200), (71, 33))
    cache, lse = check_attn(st)
    check_weights(st, cache, lse, with_in=False)


def masks_of(st, kinds):
    m = {}
    if "bias" in kinds:
        m["slopes"] = torch.tensor([2.0 ** -(i % 7) for i in range(st.h)])
    if "prefix" in kinds:
        m["prefix"] = torch.tensor([(37 * (b + 1)) % (s + 9) for b, s in enumerate(st.lens)], dtype=torch.int32)
    if "docs" in kinds:
        first = [torch.clamp((torch.arange(s - n, s) // 29) * 29, min=0) for s, n in zip(st.lens, st.new)]
        m["first"] = torch.cat(first + [torch.zeros(st.total - int(st.cu[-1]), dtype=torch.long)]).int()
    if "window" in kinds:
        first = [torch.clamp(torch.arange(s - n, s) - 40, min=0) for s, n in zip(st.lens, st.new)]
        m["first"] = torch.cat(first + [torch.zeros(st.total - int(st.cu[-1]), dtype=torch.long)]).int()
    return m


@pytest.mark.parametrize("kinds", [("bias",), ("prefix",), ("docs",), ("window", "bias"), ("prefix", "docs"), ("bias", "prefix", "docs")],
                         ids="+".join)
@pytest.mark.parametrize("cap", [0.0, 5.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masks_cap_and_bias(kinds, cap, dtype):
    st = O.Setup(len(kinds) * 10 + int(cap), dtype, 8, 2, 16, (330, 77, 150), (200, 1, 150), behind=3, q_scale=2.0)
    masks = masks_of(st, kinds)
    cache, lse = check_attn(st, cap=cap, **masks)
    check_weights(st, cache, lse, cap=cap, decay=0.5, **masks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_see_nothing(dtype):
    """First keys behind the token (and one behind every key), a table without pages: zeros and -inf, and no weight."""
    st = O.Setup(3, dtype, 4, 1, 16, (90, 40), (90, 5))
    first = torch.zeros(st.total, dtype=torch.int32)
    first[10:20] = 50
    first[70] = 2 ** 31 - 1
    st.table[1] = -1
    cache, lse = check_attn(st, first=first)
    out, _ = run_attn(st, cache, first=first)
    assert not out[10:20].any() and not out[70].any() and not out[90:].any()
    check_weights(st, cache, lse, first=first)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [-1, -2 ** 31, 2 ** 31 - 1, "pool"])
def test_pages_that_are_none(dtype, bad):
    """Keys of such pages are seen by no token; single tokens, chunks and runs of keys alike."""
    st = O.Setup(4, dtype, 8, 2, 16, (200, 900, 33), (60, 1, 33))
    for b, cols in ((0, (0, 3, 4, 5, 6, 11)), (1, (7, 55)), (2, (1,))):
        for c in cols:
            st.table[b, c] = st.num_pages if bad == "pool" else bad
    cache, lse = check_attn(st)
    check_weights(st, cache, lse)


@pytest.mark.parametrize("value", [NAN, math.inf, -math.inf])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_is_not_seen_does_not_matter(value, dtype):
    """NaN and infinities behind the last key of a page, in later tokens' rows, in other documents and before a window."""
    st = O.Setup(5, dtype, 8, 2, 32, (150, 71), (100, 71))
    for b, s in enumerate(st.lens):
        last = int(st.table[b, (s - 1) // 32])
        st.k[last, :, (s - 1) % 32 + 1:] = value
        st.v[last, :, (s - 1) % 32 + 1:] = value
    free = sorted(set(range(st.num_pages)) - set(st.table[st.table >= 0].tolist()))
    st.k[free], st.v[free] = value, value
    check_attn(st)
    t = 120   # token 120 of sequence 0 and its row in the pages: the tokens before it do not see it, from 121 on its document is not theirs
    page = int(st.table[0, t // 32])
    for rows in (st.k, st.v):
        rows[page, :, t % 32, 5] = value
    first = torch.zeros(st.total, dtype=torch.int32)
    first[t + 1 - 50:100] = t + 1
    cache = cache_of(st)
    out, lse = run_attn(st, cache, first=first)
    keep = [i for i in range(st.total) if i != t - 50]
    clean = O.Setup(5, dtype, 8, 2, 32, (150, 71), (100, 71))
    want, want_lse, tol, tol_lse = O.attention(clean, first=first)
    near(out[keep], want[keep], tol[keep], "out")
    near(lse[keep], want_lse[keep], tol_lse[keep], "lse")
    w = torch.zeros((2, 2, st.cols * 32), device=DEV)
    lse[t - 50] = -math.inf
    ck.ctkvr_cache_weights(cache, dev(st.q), lse, dev(st.k), dev(st.cu), dev(st.cur), dev(st.table), None, w, first_key=dev(first))
    clean_lse = lse.cpu()
    want_w, tol_w = O.weights(clean, clean_lse, None, torch.zeros(w.shape), 1.0, first=first)
    others = [i for i in range(150) if i != t]
    near(w[0][:, others], want_w[0][:, others], tol_w[0][:, others], "weights")


@pytest.mark.parametrize("shape", ["single", "few", "turns", "rows", "many"])
@pytest.mark.parametrize("value", [NAN, math.inf])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_left_out_of_the_weights(shape, value, dtype):
    """A row of -infinity adds nothing, whatever its query holds (a batch padded with tokens of no request): in every form of the kernels."""
    if shape == "many":
        st = many(85, dtype)
    else:
        lens, new = {"single": ((500, 90, 33), (1, 1, 1)), "few": ((300, 129), (40, 3)), "turns": ((600,), (180,)), "rows": ((700,), (700,))}[shape]
        st = O.Setup(85, dtype, 8, 2, 16, lens, new, q_scale=2.0)
    cache = cache_of(st)
    _, lse = run_attn(st, cache)
    n, q = int(st.cu[-1]), dev(st.q).clone()
    out = torch.rand((n, st.h), generator=st.gen) < 0.3     # single heads,
    out[::7] = True                                         # whole tokens,
    out[-1, 1:] = True                                      # and the last rows of all
    lse[:n][out.to(DEV)] = -math.inf
    q[:n][out.to(DEV)] = value
    w_in, w = torch.rand((st.batch, st.g, st.cols * 16), generator=st.gen), torch.full((st.batch, st.g, st.cols * 16), 5.0, device=DEV)
    ck.ctkvr_cache_weights(cache, q, lse, dev(st.k), dev(st.cu), dev(st.cur), dev(st.table), dev(w_in), w, decay=0.5)
    want, tol = O.weights(st, lse.cpu(), w_in, torch.full(w.shape, 5.0), 0.5)
    near(w, want, tol, "weights")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_that_are_seen_and_not_finite(dtype):
    """An infinite value reaches the rows that see its key, in its column, and no others."""
    st = O.Setup(6, dtype, 4, 2, 16, (100,), (100,))
    page = int(st.table[0, 40 // 16])
    st.v[page, 1, 40 % 16, 9] = math.inf
    st.v[page, 1, 40 % 16, 70] = NAN
    out, lse = run_attn(st, cache_of(st))
    assert torch.isfinite(lse).all() and torch.isfinite(out[:40]).all() and torch.isfinite(out[:, :2]).all()
    assert (out[40:, 2:, 9] == math.inf).all() and torch.isnan(out[40:, 2:, 70]).all()
    rest = [d for d in range(128) if d not in (9, 70)]
    assert torch.isfinite(out[:, :, rest]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_views_of_a_fused_projection_and_unequal_strides(dtype):
    st = O.Setup(7, dtype, 8, 2, 16, (70, 90), (70, 40))
    fused = torch.full((st.total, 12 * 128 + 64), NAN, dtype=st.td, device=DEV)
    q = fused[:, :8 * 128].view(st.total, 8, 128)
    q.copy_(st.q)
    cache = cache_of(st)
    a, la = run_attn(st, cache, q=q)
    b, lb = run_attn(st, cache)
    assert torch.equal(a, b) and torch.equal(la, lb)
    w1, w2 = (torch.zeros((2, 2, st.cols * 16), device=DEV) for _ in range(2))
    for qq, w in ((q, w1), (dev(st.q), w2)):
        ck.ctkvr_cache_weights(cache, qq, la, dev(st.k), dev(st.cu), dev(st.cur), dev(st.table), None, w)
    assert torch.equal(w1, w2)


def test_scores_that_are_large():
    """Scores of several thousand, apart by more than an exponent holds: the maximum runs with the keys, also where keys are split."""
    for new in (1, 40):
        st = O.Setup(8, "f32", 4, 1, 16, (2000,), (new,), q_scale=300.0)
        st.k = (st.k * 20).to(st.td)
        out, lse = run_attn(st, cache_of(st))
        want, want_lse, _, _ = O.attention(st)
        # scores of 10^5 have fp32 steps of 2^-7: two keys that far apart may trade places, a single winner may not
        z, _ = O.scores(st, 0)
        top = z.topk(2, dim=-1).values
        clear = ((top[..., 0] - top[..., 1]) > 30).permute(2, 0, 1).reshape(new, 4)
        assert clear.float().mean() > 0.9
        got, want = out.cpu().double()[clear], want[clear]
        assert torch.isfinite(out).all() and ((got - want).abs() <= 2.0 ** -20 * want.abs() + 1e-6).all()
        assert ((lse.cpu().double() - want_lse).abs() <= 140 * 2.0 ** -23 * want_lse.abs().max() * 2).all()


def test_a_cache_beyond_32_bit_offsets():
    """Rows whose byte and element offsets pass 2^32."""
    g, page, pool = 8, 16, 280000                   # 2^32 elements are 262144 pages
    st = O.Setup(9, "bf16", 8, g, page, (100,), (30,))
    big = []
    for small in (st.k, st.v):
        t = torch.empty((pool, g, page, 128), dtype=torch.bfloat16, device=DEV)
        used = st.table[0, :7].long()
        t[(pool - 1 - used).to(DEV)] = small[used].to(DEV)
        big.append(t)
    table = torch.where(st.table >= 0, pool - 1 - st.table, -1).to(DEV)
    cache = cache_of(st, num_pages=pool)
    out, lse = torch.empty((30, 8, 128), dtype=torch.bfloat16, device=DEV), torch.empty((30, 8), device=DEV)
    ck.ctkvr_cache_attn(cache, dev(st.q), *big, dev(st.cu), dev(st.cur), table, out, out_lse=lse)
    want, want_lse, tol, tol_lse = O.attention(st)
    near(out, want, tol, "out")
    w = torch.zeros((1, g, st.cols * page), device=DEV)
    ck.ctkvr_cache_weights(cache, dev(st.q), lse, big[0], dev(st.cu), dev(st.cur), table, None, w)
    want_w, tol_w = O.weights(st, lse.cpu(), None, torch.zeros(w.shape), 1.0)
    near(w, want_w, tol_w, "weights")
    kn = torch.randn((30, g, 128), generator=st.gen).bfloat16().to(DEV)
    ck.ctkvr_cache_append(cache, None, kn, kn, dev(st.cu), dev(st.cur), table, None, *big)
    ids = torch.zeros((1, g, 50), dtype=torch.int32, device=DEV)
    ck.ctkvr_cache_evict(cache, w, *big, dev(st.cur), table, 50, ids, n_local=30)
    for i in (0, 19, 20, 49):                        # the last 30 tokens are the appended ones
        t = int(ids[0, 0, i])
        row = big[1][table[0, i // page].long(), 0, i % page].cpu()
        assert torch.equal(row, kn[t - 70, 0].cpu() if t >= 70 else st.v[int(st.table[0, t // page]), 0, t % page])


# ---- forms of the kernels that larger calls take: rows of 128 a block, keys split or not, rows past the keys ----------------
def many(seed, dtype, h=32, g=8, page=16, q_scale=1.5):
    """16 sequences with enough new tokens that rows are taken 128 at a time and, for the weights, past the keys."""
    r = np.random.RandomState(seed)
    lens = [int(x) for x in r.randint(150, 420, size=16)]
    new = [min(s, int(x)) for s, x in zip(lens, r.randint(140, 190, size=16))]
    lens[3], new[3] = 64, 64
    lens[5], new[5] = 300, 1
    lens[7], new[7] = 0, 0
    lens[8], new[8] = 129, 0
    lens[9], new[9] = 400, 400
    return O.Setup(seed, dtype, h, g, page, lens, new, behind=2, q_scale=q_scale)


@pytest.mark.parametrize("kinds", [(), ("bias",), ("prefix",), ("docs",), ("window", "prefix", "bias")], ids=lambda k: "+".join(k) or "causal")
@pytest.mark.parametrize("cap", [0.0, 4.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows(kinds, cap, dtype):
    st = many(51 + len(kinds), dtype)
    masks = masks_of(st, kinds)
    cache, lse = check_attn(st, cap=cap, **masks)
    check_weights(st, cache, lse, cap=cap, decay=0.75, **masks)


@pytest.mark.parametrize("page", [1, 4, 64, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows_page_sizes_and_pages_that_are_none(page, dtype):
    st = many(60 + page, dtype, page=page)
    for b in (0, 4, 9):
        cols = [c for c in (0, 1, 5, 70, 71) if c < -(-st.lens[b] // page)][:3]
        for c in cols:
            st.table[b, c] = st.num_pages if c % 2 else -1
    cache, lse = check_attn(st)
    check_weights(st, cache, lse, with_in=False)


@pytest.mark.parametrize("value", [NAN, math.inf])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows_what_is_not_seen(value, dtype):
    st, clean = many(71, dtype, h=8, g=8), many(71, dtype, h=8, g=8)
    first = torch.zeros(st.total, dtype=torch.int32)
    hidden = []
    for b in (1, 9, 12):                     # one token's row is hidden from all others of its sequence: the earlier ones by position
        s, n = st.lens[b], st.new[b]
        t = s - n // 2
        hidden.append(int(st.cu[b]) + n - n // 2)
        for rows in (st.k, st.v):
            rows[int(st.table[b, t // 16]), :, t % 16, 3:70:9] = value
        first[hidden[-1] + 1:int(st.cu[b + 1])] = t + 1
    for b, s in enumerate(st.lens):
        if s % 16:
            for rows in (st.k, st.v):
                rows[int(st.table[b, (s - 1) // 16]), :, s % 16:] = value
    out, lse = run_attn(st, cache_of(st), first=first)
    want, want_lse, tol, tol_lse = O.attention(clean, first=first)
    keep = [i for i in range(int(st.cu[-1])) if i not in hidden]
    near(out[keep], want[keep], tol[keep], "out")
    near(lse[keep], want_lse[keep], tol_lse[keep], "lse")


@pytest.mark.parametrize("cap", [0.0, 5.0])
@pytest.mark.parametrize("lens,new,h,g", [((4300, 5000), (140, 131), 8, 1), ((6000,), (70,), 16, 2)])
def test_many_rows_with_their_keys_split(lens, new, h, g, cap):
    st = O.Setup(81, "bf16", h, g, 16, lens, new, q_scale=2.0)
    check_attn(st, cap=cap, **masks_of(st, ("prefix", "bias")))
    check_attn(st, cap=cap, **masks_of(st, ("window",)))


@pytest.mark.parametrize("scale", [0.5, 40.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_around_the_cap(scale, dtype):
    """Below the cap and far beyond it, in one call."""
    st = O.Setup(82, dtype, 8, 2, 16, (200, 90), (100, 1), q_scale=scale)
    cache, lse = check_attn(st, cap=2.0)
    check_weights(st, cache, lse, cap=2.0)


@pytest.mark.parametrize("shape", ["few", "many"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_capped_scores_are_a_matter_of_their_own_size(shape, bias, dtype):
    """A token whose scores are far beyond the cap: the tokens before it, which do not see its key, and all keys' weights without its row are the
    same to the bit."""
    st = many(84, dtype, q_scale=1.0) if shape == "many" else O.Setup(84, dtype, 4, 2, 16, (200, 90, 700), (100, 90, 2))
    masks = masks_of(st, ("bias",)) if bias else {}
    slopes = dev(masks.get("slopes"))
    loud = [int(st.cu[b + 1]) - 1 for b, n in enumerate(st.new) if n > 1]
    quiet = [i for i in range(int(st.cu[-1])) if i not in loud]
    got = []
    for factor in (1.0, 100.0):
        q, k = st.q.clone(), st.k.clone()
        q[loud] *= factor
        for b, n in enumerate(st.new):
            if n > 1:
                t = st.lens[b] - 1
                k[int(st.table[b, t // 16]), :, t % 16] *= factor
        cache = cache_of(st, softcap=30.0)
        out, lse = torch.zeros((st.total, st.h, 128), dtype=st.td, device=DEV), torch.zeros((st.total, st.h), device=DEV)
        ck.ctkvr_cache_attn(cache, dev(q), dev(k), dev(st.v), dev(st.cu), dev(st.cur), dev(st.table), out, out_lse=lse, slopes=slopes)
        w, only = torch.zeros((st.batch, st.g, st.cols * 16), device=DEV), lse.clone()
        only[loud] = -math.inf
        ck.ctkvr_cache_weights(cache, dev(q), only, dev(k), dev(st.cu), dev(st.cur), dev(st.table), None, w, slopes=slopes)
        got.append((out[quiet], lse[quiet], w))
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_few_rows_joined_in_the_launch_and_replayed(dtype):
    """One sequence's single token over many keys: the runs' hand-over, in eager calls and in two graphs on one handle that take turns."""
    st = O.Setup(83, dtype, 4, 1, 16, (3000,), (1,), q_scale=2.0)
    cache, _ = check_attn(st)
    want, want_lse, tol, tol_lse = O.attention(st)
    args = [dev(x) for x in (st.k, st.v, st.cu, st.cur, st.table)]
    q = dev(st.q).clone()
    outs = [(torch.zeros((1, 4, 128), dtype=st.td, device=DEV), torch.zeros((1, 4), device=DEV)) for _ in range(2)]
    graphs = []
    torch.cuda.synchronize()
    for o, l in outs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            ck.ctkvr_cache_attn(cache, q, *args, o, out_lse=l)
    first = None
    for i in range(6):
        o, l = outs[i % 2]
        o.zero_(), l.zero_()
        graphs[i % 2].replay()
        near(o, want, tol, "out")
        near(l, want_lse, tol_lse, "lse")
        eager = torch.zeros_like(o)
        ck.ctkvr_cache_attn(cache, q, *args, eager)
        first = o.clone() if first is None else first
        assert torch.equal(o, first) and torch.equal(eager, first)


def test_weights_of_a_large_batch_with_a_wide_table():
    """Blocks for every 128 keys of 1024 sequences' tables of 2^17 tokens are 2^32 threads.  The sequences are one, again and again."""
    batch, n, page = 1024, 300, 256
    one = O.Setup(86, "f32", 8, 8, page, (n,), (n,), q_scale=2.0)
    q = dev(one.q).repeat(batch, 1, 1)
    table = torch.full((batch, 512), -1, dtype=torch.int32, device=DEV)
    table[:, :2] = dev(one.table[0, :2])
    cu = (n * torch.arange(batch + 1, device=DEV)).int()
    cur = torch.full((batch,), n, dtype=torch.int32, device=DEV)
    cache = ck.ctkvr_cache_create(ck.CacheParams(batch=batch, n_q_heads=8, n_kv_heads=8, num_pages=one.num_pages, max_pages=512, max_new=batch * n,
                                                 page_size=page, dtype=ck.F32))
    lse = run_attn(one, cache_of(one))[1]
    w = torch.full((batch, 8, 512 * page), 5.0, device=DEV)
    ck.ctkvr_cache_weights(cache, q, lse.repeat(batch, 1), dev(one.k), cu, cur, table, None, w)
    want, tol = O.weights(one, lse.cpu(), None, torch.full((1, 8, n), 5.0), 1.0)
    near(w[:1, :, :n], want, tol, "weights")
    assert (w[:, :, :n] == w[:1, :, :n]).all() and (w[:, :, n:] == 5).all()


@pytest.mark.parametrize("scale", [0.02, 0.31])
@pytest.mark.parametrize("cap", [0.0, 4.0])
@pytest.mark.parametrize("shape", ["few", "rows", "many"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_scale_of_ones_own(shape, cap, scale, dtype):
    if shape == "many":
        st = many(87, dtype)
    else:
        lens, new = {"few": ((300, 900, 50), (40, 1, 50)), "rows": ((600,), (600,))}[shape]
        st = O.Setup(87, dtype, 8, 2, 16, lens, new, behind=2)
    slopes = torch.tensor([2.0 ** -(i % 9 + 2) for i in range(st.h)])
    for bias in (None, slopes):
        cache = cache_of(st, softcap=cap, sm_scale=scale)
        out, lse = run_attn(st, cache, slopes=bias)
        n = int(st.cu[-1])
        want, want_lse, tol, tol_lse = O.attention(st, cap=cap, slopes=bias, scale=float(np.float32(scale)))
        near(out[:n], want, tol, "out")
        near(lse[:n], want_lse, tol_lse, "lse")
        check_weights(st, cache, lse, cap=cap, decay=0.5, slopes=bias, scale=float(np.float32(scale)))


@pytest.mark.parametrize("batch", [65, 130])
@pytest.mark.parametrize("new", [1, 20, 70])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_sequences_than_a_wave_has_lanes(batch, new, dtype):
    """Sequences are looked up 64 at a time: empty ones and ones without new tokens around there, single tokens, chunks and prompts."""
    r = np.random.RandomState(batch + new)
    lens = [int(x) for x in r.randint(new, new + 60, size=batch)]
    news = [new if new == 1 else int(x) for x in r.randint(new // 2 + 1, new + 1, size=batch)]
    for b in (0, 62, 64, batch - 2):
        news[b] = 0
    lens[62], lens[3], lens[batch - 1] = 0, 3000, 2000
    st = O.Setup(88, dtype, 8, 2, 16, lens, news, behind=3, q_scale=2.0)
    cache, lse = check_attn(st)
    check_weights(st, cache, lse, decay=0.75)
    kn, vn = (torch.randn((st.total, 2, 128), generator=st.gen).to(st.td).to(DEV) for _ in range(2))
    freq = 10000.0 ** (-np.arange(64) / 64.0)
    k, v, n, slots, pos = check_append(st, cache, freq, np.zeros(64, int), None, None, kn, vn)
    wk, tk = O.rotated(kn[:n].cpu(), pos, freq, np.zeros(64, int))
    full_k, full_v, tol_k = st.k.to(O.F8), st.v.clone(), torch.zeros_like(st.k, dtype=O.F8)
    pages = st.table[torch.repeat_interleave(torch.arange(batch), torch.tensor(news)), slots // 16].long()
    full_k[pages, :, slots % 16], full_v[pages, :, slots % 16] = wk, vn[:n].cpu()
    tol_k[pages, :, slots % 16] = tk + wk.abs() * O.HALF[dtype]
    near(k, full_k, tol_k, "k_pages")
    assert torch.equal(v.cpu(), full_v), "v_pages"


@pytest.mark.parametrize("lens,new,h,g", [
    ((1500,) + (40, 3000, 700, 1) * 4, (1024,) + (1,) * 16, 8, 2),        # the weights' rows in several turns
    ((700, 9000, 5000, 33), (600, 1, 1, 1), 8, 2),                        # rows of 128, keys split
    ((300, 5000, 1300, 4000), (1, 1, 1100, 1), 32, 8),                    # ... not split
], ids=["turns", "split", "whole"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_chunk_beside_single_tokens(lens, new, h, g, dtype):
    st = O.Setup(89, dtype, h, g, 16, lens, new, behind=1, q_scale=2.0)
    cache, lse = check_attn(st)
    check_weights(st, cache, lse, decay=0.75)
    masks = masks_of(st, ("window", "prefix", "bias"))
    cache, lse = check_attn(st, cap=5.0, **masks)
    check_weights(st, cache, lse, cap=5.0, **masks)


# ---- append ----------------------------------------------------------------------------------------------------
def check_append(st, cache, freq, axis, positions, q=None, kn=None, vn=None, q_out=None):
    k, v = dev(st.k).clone(), dev(st.v).clone()
    ck.ctkvr_cache_append(cache, q, kn, vn, dev(st.cu), dev(st.cur), dev(st.table), q_out, k if kn is not None else None,
                          v if kn is not None else None, positions=dev(positions))
    n = int(st.cu[-1])
    slots = torch.cat([torch.arange(s - m, s) for s, m in zip(st.lens, st.new)])
    pos = positions[:, :n] if positions is not None else slots[None].expand(3, -1)
    return k, v, n, slots, pos


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("axes", [1, 3])
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("h,g,page", [(8, 2, 16), (4, 4, 1), (40, 10, 64)])
def test_append(dtype, axes, given, h, g, page):
    st = O.Setup(11, dtype, h, g, page, (40, 1, 0, 130), (17, 1, 0, 65), behind=2)
    axis = np.arange(64) % 3 if axes == 3 else np.zeros(64, int)
    freq = 10000.0 ** (-np.arange(64) / 64.0)
    positions = None
    if given:
        positions = torch.randint(-100, 200000, (axes, st.total), generator=st.gen).int()
        positions[:, 0], positions[:, 1], positions[:, 2] = 2 ** 31 - 1, -2 ** 31, 0
    fused = torch.randn((st.total, (h + 2 * g) * 128), generator=st.gen).to(st.td).to(DEV)
    q, kn, vn = (t.view(st.total, -1, 128) for t in torch.split(fused, [h * 128, g * 128, g * 128], dim=1))
    q_out = torch.full((st.total, h, 128), 7.0, dtype=st.td, device=DEV)
    cache = cache_of(st, rope_axis=axis if axes == 3 else None)
    k, v, n, slots, pos = check_append(st, cache, freq, axis, positions, q, kn, vn, q_out)
    want, tol = O.rotated(q[:n].cpu(), pos, freq, axis)
    near(q_out[:n], want, tol + want.abs() * O.HALF[dtype], "q")
    assert (q_out[n:] == 7).all()
    wk, tk = O.rotated(kn[:n].cpu(), pos, freq, axis)
    full_k, full_v, tol_k = st.k.to(O.F8), st.v.clone(), torch.zeros_like(st.k, dtype=O.F8)
    b = torch.cat([torch.full((m,), i) for i, m in enumerate(st.new)]).long()
    pages = st.table[b, slots // page].long()
    full_k[pages, :, slots % page] = wk
    tol_k[pages, :, slots % page] = tk + wk.abs() * O.HALF[dtype]
    full_v[pages, :, slots % page] = vn[:n].cpu()
    near(k, full_k, tol_k, "k_pages")
    assert torch.equal(v.cpu(), full_v), "v_pages"


def test_append_with_frequencies_of_ones_own_in_place_and_in_parts():
    """Given frequencies (some zero: not rotated, some above a turn a token), q rotated where it is, q alone and k and v alone."""
    st = O.Setup(12, "f32", 8, 2, 16, (50,), (20,))
    freq = np.where(np.arange(64) < 40, 1.0 / (1.0 + np.arange(64)) ** 2, 0.0)
    freq[3] = 7.5
    cache = cache_of(st, rope_freq=freq)
    kn, vn = (torch.randn((20, 2, 128), generator=st.gen).to(DEV) for _ in range(2))
    q = dev(st.q).clone()
    k, v, n, slots, pos = check_append(st, cache, freq, np.zeros(64, int), None, q, None, None, q)
    assert torch.equal(k.cpu(), st.k) and torch.equal(v.cpu(), st.v)
    want, tol = O.rotated(st.q, pos, freq, np.zeros(64, int))
    near(q, want, tol + want.abs() * O.HALF["f32"], "q in place")
    assert torch.equal(q.cpu()[..., 40:64], st.q[..., 40:64]) and torch.equal(q.cpu()[..., 104:], st.q[..., 104:])
    k, v, n, slots, pos = check_append(st, cache, freq, np.zeros(64, int), None, None, kn, vn)
    wk, tk = O.rotated(kn.cpu(), pos, freq, np.zeros(64, int))
    pages = st.table[0, slots // 16].long()
    near(k[pages.to(DEV), :, (slots % 16).to(DEV)], wk, tk + wk.abs() * O.HALF["f32"], "k alone")
    assert torch.equal(v[pages.to(DEV), :, (slots % 16).to(DEV)], vn)


def test_append_into_slots_and_pages_that_are_none():
    """Tokens beyond the table, before slot 0 and on bad pages are dropped; everything else is written, and nothing else."""
    st = O.Setup(13, "bf16", 4, 2, 16, (64, 30, 40), (10, 30, 5), spare_cols=0)
    st.cur = torch.tensor([68, 20, 40], dtype=torch.int32)     # 4 tokens beyond 64 slots; 10 before slot 0
    st.table[2, 2] = st.num_pages
    kn = torch.randn((45, 2, 128), generator=st.gen).bfloat16().to(DEV)
    cache = cache_of(st)
    k, v = dev(st.k).clone(), dev(st.v).clone()
    ck.ctkvr_cache_append(cache, None, kn, kn, dev(st.cu), dev(st.cur), dev(st.table), None, k, v)
    want = st.v.clone()
    for b, (c0, n) in enumerate(((0, 10), (10, 30), (40, 5))):
        for i in range(n):
            slot = int(st.cur[b]) - n + i
            if 0 <= slot < st.cols * 16 and 0 <= int(st.table[b, slot // 16]) < st.num_pages:
                want[int(st.table[b, slot // 16]), :, slot % 16] = kn[c0 + i].cpu()
    assert torch.equal(v.cpu(), want)
    changed = (k.cpu() != st.k).any(dim=-1)
    assert torch.equal(changed, (want != st.v).any(dim=-1))


# ---- eviction ----------------------------------------------------------------------------------------------------
EVICT = [
    # lens, budget, n_init, n_local
    ((100, 40, 0, 1), 50, 0, 0), ((100, 51, 50, 49), 50, 4, 10), ((1000, 333), 1, 0, 0), ((1000, 333), 1, 1, 0), ((1000, 333), 300, 0, 300),
    ((70, 700), 64, 32, 32), ((3000, 2049), 2048, 4, 100), ((5000,), 17, 3, 5), ((2100, 1030, 1025), 1024, 0, 1), ((40,), 4000, 5, 5),
]


@pytest.mark.parametrize("case", EVICT, ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("values", ["spread", "ties", "equal", "odd"])
def test_evict(case, dtype, values):
    lens, budget, n_init, n_local = case
    st = O.Setup(21, dtype, 4, 2, 16, lens, (0,) * len(lens))
    w = torch.rand((st.batch, 2, st.cols * 16), generator=st.gen)
    if values == "ties":
        w = (w * 5).floor()
    elif values == "equal":
        w[:] = 0.25
    elif values == "odd":                       # both zeros, NaN, infinities, negative and subnormal values
        pick = torch.tensor([0.0, -0.0, NAN, math.inf, -math.inf, -1.0, 1e-40, -1e-40, 3.0])
        w = pick[torch.randint(0, 9, w.shape, generator=st.gen)]
    ids, lens_out, w_want, k_want, v_want = O.evicted(st, w, budget, n_init, n_local)
    for in_place in (False, True):
        k, v, wd = dev(st.k).clone(), dev(st.v).clone(), dev(w).clone()
        w_out = wd if in_place else torch.full_like(wd, 9.0)
        got = torch.full((st.batch, 2, budget), 77, dtype=torch.int32, device=DEV)
        kept = torch.zeros(st.batch, dtype=torch.int32, device=DEV)
        ck.ctkvr_cache_evict(cache_of(st), wd, k, v, dev(st.cur), dev(st.table), budget, got, n_init=n_init, n_local=n_local, weights_out=w_out,
                             out_lens=kept)
        assert kept.tolist() == lens_out
        assert np.array_equal(got.cpu().numpy(), ids)
        assert torch.equal(k.cpu(), k_want) and torch.equal(v.cpu(), v_want)
        for b, m in enumerate(lens_out):
            assert np.array_equal(w_out[b, :, :m].cpu().numpy(), w_want[b, :, :m].numpy(), equal_nan=True)
            rest = (w[b, :, m:] if in_place else torch.full_like(w[b, :, m:], 9.0)).numpy()
            assert np.array_equal(w_out[b, :, m:].cpu().numpy(), rest, equal_nan=True)


@pytest.mark.parametrize("lens", [(20000, 9000), (50000, 33000), (70000, 65537)], ids=str)
@pytest.mark.parametrize("values", ["spread", "narrow", "ties", "equal"])
def test_evict_from_long_sequences(lens, values):
    """Every number of ranks that a thread of the selection holds, none among them, and more weights that agree than shared memory has room for."""
    st = O.Setup(23, "bf16", 1, 1, 64, lens, (0, 0))
    w = torch.rand((2, 1, st.cols * 64), generator=st.gen)
    if values == "narrow":                     # one bin of the first round
        w = 1.0 + w / 4096
    elif values == "ties":
        w = (w * 5).floor()
    elif values == "equal":
        w[:] = 2.0
    for budget, n_init, n_local in ((700, 4, 100), (12000, 0, 1)):
        ids, lens_out, w_want, k_want, v_want = O.evicted(st, w, budget, n_init, n_local)
        k, v, w_out = dev(st.k).clone(), dev(st.v).clone(), torch.zeros_like(w, device=DEV)
        got = torch.zeros((2, 1, budget), dtype=torch.int32, device=DEV)
        ck.ctkvr_cache_evict(cache_of(st), dev(w), k, v, dev(st.cur), dev(st.table), budget, got, n_init=n_init, n_local=n_local, weights_out=w_out)
        assert np.array_equal(got.cpu().numpy(), ids)
        assert torch.equal(k.cpu(), k_want) and torch.equal(v.cpu(), v_want) and torch.equal(w_out.cpu(), w_want)


def test_evict_with_pages_that_are_none():
    st = O.Setup(22, "bf16", 4, 2, 16, (500, 300), (0, 0))
    st.table[0, 3], st.table[0, 20], st.table[1, 0], st.table[1, 18] = -1, st.num_pages, -7, 2 ** 31 - 1
    w = torch.rand((2, 2, st.cols * 16), generator=st.gen)
    ids, lens_out, _, k_want, v_want = O.evicted(st, w, 100, 3, 40)
    k, v = dev(st.k).clone(), dev(st.v).clone()
    got = torch.zeros((2, 2, 100), dtype=torch.int32, device=DEV)
    ck.ctkvr_cache_evict(cache_of(st), dev(w), k, v, dev(st.cur), dev(st.table), 100, got, n_init=3, n_local=40)
    assert np.array_equal(got.cpu().numpy(), ids)
    assert torch.equal(k.cpu(), k_want) and torch.equal(v.cpu(), v_want)


def test_evict_with_the_lengths_written_in_place():
    """out_lens is cur_lens: every head and the move see the lengths before, eagerly and in a captured call whose lengths are set again."""
    st = O.Setup(24, "bf16", 8, 8, 16, (700, 50, 0, 1300, 81, 80, 900, 1299), (0,) * 8)
    w = torch.rand((8, 8, st.cols * 16), generator=st.gen)
    ids, lens_out, w_want, k_want, v_want = O.evicted(st, w, 80, 4, 16)
    k, v, wd, cur, table = dev(st.k).clone(), dev(st.v).clone(), dev(w).clone(), dev(st.cur).clone(), dev(st.table)
    got, cache = torch.full((8, 8, 80), 77, dtype=torch.int32, device=DEV), cache_of(st)

    def call():
        ck.ctkvr_cache_evict(cache, wd, k, v, cur, table, 80, got, n_init=4, n_local=16, weights_out=wd, out_lens=cur)

    def check():
        assert cur.tolist() == lens_out
        assert np.array_equal(got.cpu().numpy(), ids)
        assert torch.equal(k.cpu(), k_want) and torch.equal(v.cpu(), v_want)
        for b, m in enumerate(lens_out):
            assert torch.equal(wd[b, :, :m].cpu(), w_want[b, :, :m])

    call()
    check()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call()
    for _ in range(4):
        k.copy_(st.k), v.copy_(st.v), wd.copy_(w), cur.copy_(st.cur), got.fill_(77)
        graph.replay()
        check()


# ---- streams, graphs, repetition -----------------------------------------------------------------------------------
@pytest.mark.parametrize("new", [1, 90])
def test_the_same_call_gives_the_same_bits_on_any_stream(new):
    st = O.Setup(31, "bf16", 8, 2, 16, (3000, 700), (new, new))
    cache = cache_of(st)
    out, lse = run_attn(st, cache)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again, lse2 = run_attn(st, cache)
    torch.cuda.synchronize()
    assert torch.equal(out, again) and torch.equal(lse, lse2)


def test_captured_steps_replay_with_lengths_that_have_changed():
    """A decode step (append, attention, weights) captured once and replayed as the sequences grow, with eager work in between, against
    the same steps run eagerly."""
    st = O.Setup(32, "bf16", 8, 2, 16, (200, 331), (1, 1), spare_cols=2)
    st.table[0, 13:15] = torch.tensor([st.num_pages, st.num_pages + 1], dtype=torch.int32)
    st.table[1, 21:23] = torch.tensor([st.num_pages + 2, st.num_pages + 3], dtype=torch.int32)
    st.num_pages += 4
    st.k, st.v = (torch.cat([x, torch.zeros((4,) + x.shape[1:], dtype=x.dtype)]) for x in (st.k, st.v))
    width = st.cols * 16
    steps = 12
    qs, ks, vs = (torch.randn((steps, 2, n, 128), generator=st.gen).bfloat16().to(DEV) for n in (8, 2, 2))

    def state():
        return {"q": torch.zeros((2, 8, 128), dtype=torch.bfloat16, device=DEV), "kn": torch.zeros((2, 2, 128), dtype=torch.bfloat16, device=DEV),
                "vn": torch.zeros((2, 2, 128), dtype=torch.bfloat16, device=DEV), "k": dev(st.k).clone(), "v": dev(st.v).clone(),
                "cur": dev(st.cur).clone(), "w": torch.zeros((2, 2, width), device=DEV), "lse": torch.zeros((2, 8), device=DEV),
                "out": torch.zeros((2, 8, 128), dtype=torch.bfloat16, device=DEV), "cu": dev(st.cu), "table": dev(st.table), "cache": cache_of(st)}

    def step(s):
        ck.ctkvr_cache_append(s["cache"], s["q"], s["kn"], s["vn"], s["cu"], s["cur"], s["table"], s["q"], s["k"], s["v"])
        ck.ctkvr_cache_attn(s["cache"], s["q"], s["k"], s["v"], s["cu"], s["cur"], s["table"], s["out"], out_lse=s["lse"])
        ck.ctkvr_cache_weights(s["cache"], s["q"], s["lse"], s["k"], s["cu"], s["cur"], s["table"], s["w"], s["w"], decay=0.9)

    def load(s, i):
        s["q"].copy_(qs[i]), s["kn"].copy_(ks[i]), s["vn"].copy_(vs[i])
        s["cur"].copy_(st.cur + i)

    eager, graphed = state(), state()
    warm = state()
    load(warm, 0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(warm)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(graphed)
    for i in range(steps):
        load(eager, i)
        step(eager)
        load(graphed, i)
        graph.replay()
        for name in ("out", "lse", "w", "k", "v"):
            assert torch.equal(eager[name], graphed[name]), (i, name)


def test_captured_eviction_replays():
    st = O.Setup(33, "bf16", 4, 2, 16, (700, 90), (0, 0))
    cache, ids = cache_of(st), torch.zeros((2, 2, 80), dtype=torch.int32, device=DEV)
    w, k, v = torch.zeros((2, 2, st.cols * 16), device=DEV), dev(st.k).clone(), dev(st.v).clone()
    kept, cur, table = torch.zeros(2, dtype=torch.int32, device=DEV), dev(st.cur), dev(st.table)
    ck.ctkvr_cache_evict(cache, w, k, v, cur, table, 80, ids, n_init=2, n_local=9, weights_out=w, out_lens=kept)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        ck.ctkvr_cache_evict(cache, w, k, v, cur, table, 80, ids, n_init=2, n_local=9, weights_out=w, out_lens=kept)
    for i in range(4):
        fresh = torch.rand(w.shape, generator=st.gen)
        w.copy_(fresh), k.copy_(st.k), v.copy_(st.v)
        graph.replay()
        want_ids, lens, w_want, k_want, v_want = O.evicted(st, fresh, 80, 2, 9)
        assert np.array_equal(ids.cpu().numpy(), want_ids) and kept.tolist() == lens
        assert torch.equal(k.cpu(), k_want) and torch.equal(v.cpu(), v_want) and torch.equal(w.cpu()[:, :, :80], w_want[:, :, :80])


# ---- together -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_prompt_in_chunks_then_a_smaller_cache_then_an_index_on_it(dtype):
    """Two prompts enter in chunks (append, attention, weights), the cache is cut down, and an index built on what is left serves a decode step
    with every centroid probed, so that it attends over the whole of the smaller cache."""
    h, g, page, lens, budget = 8, 2, 16, (300, 220), 128
    chunks = ((100, 130), (150, 1), (50, 89))
    r = torch.Generator().manual_seed(77)
    base = O.Setup(41, dtype, h, g, page, lens, (0, 0))
    cache = cache_of(base, max_new=300)
    k, v, table = dev(base.k).zero_(), dev(base.v).zero_(), dev(base.table)
    w = torch.zeros((2, g, base.cols * page), device=DEV)
    k_all, v_all = dev(base.k), dev(base.v)
    done, q_tail = [0, 0], [[], []]
    freq = 10000.0 ** (-np.arange(64) / 64.0)
    for new in chunks:
        done = [d + n for d, n in zip(done, new)]
        total = sum(new)
        cu, cur = torch.tensor([0, new[0], total], dtype=torch.int32), torch.tensor(done, dtype=torch.int32)
        q, kn, vn = (torch.randn((total, n, 128), generator=r).to(base.td) for n in (h, g, g))
        q_dev = torch.empty((total, h, 128), dtype=base.td, device=DEV)
        out, lse = torch.empty_like(q_dev), torch.empty((total, h), device=DEV)
        ck.ctkvr_cache_append(cache, dev(q), dev(kn), dev(vn), dev(cu), dev(cur), table, q_dev, k, v)
        ck.ctkvr_cache_attn(cache, q_dev, k, v, dev(cu), dev(cur), table, out, out_lse=lse)
        before = w.clone()
        ck.ctkvr_cache_weights(cache, q_dev, lse, k, dev(cu), dev(cur), table, w, w)
        # the step against the oracle on the rows that the append has left
        st = O.Setup(41, dtype, h, g, page, lens, (0, 0))
        st.lens, st.new, st.cu, st.cur, st.total = done, list(new), cu, cur, total
        st.q, st.k, st.v = q_dev.cpu(), k.cpu(), v.cpu()
        pos = torch.cat([torch.arange(d - n, d) for d, n in zip(done, new)])[None].expand(3, -1)
        want_q, tol_q = O.rotated(q, pos, freq, np.zeros(64, int))
        near(q_dev, want_q, tol_q + want_q.abs() * O.HALF[dtype], "q")
        want, want_lse, tol, tol_lse = O.attention(st)
        near(out, want, tol, "out")
        near(lse, want_lse, tol_lse, "lse")
        want_w, tol_w = O.weights(st, lse.cpu(), before.cpu(), before.cpu(), 1.0)
        near(w, want_w, tol_w, "weights")
        for b in range(2):
            q_tail[b].append(q_dev[int(cu[b]):int(cu[b + 1])])
    assert done == list(lens)
    # every query head's weights of a token add up to 1
    assert torch.allclose(w.sum(dim=-1).cpu(), torch.tensor([[s * h / g] * g for s in lens]), rtol=1e-5)
    st.k, st.v, st.lens, st.cur = k.cpu(), v.cpu(), list(lens), torch.tensor(lens, dtype=torch.int32)
    ids, kept, w_want, k_want, v_want = O.evicted(st, w.cpu(), budget, 4, 32)
    got, kept_dev = torch.empty((2, g, budget), dtype=torch.int32, device=DEV), torch.empty(2, dtype=torch.int32, device=DEV)
    ck.ctkvr_cache_evict(cache, w, k, v, dev(st.cur), table, budget, got, n_init=4, n_local=32, weights_out=w, out_lens=kept_dev)
    assert np.array_equal(got.cpu().numpy(), ids) and kept_dev.tolist() == [budget, budget]
    assert torch.equal(k.cpu(), k_want) and torch.equal(v.cpu(), v_want)
    C = 8
    tail = torch.cat([torch.cat(q_tail[b])[-C:] for b in range(2)]).contiguous()
    p = ck.Params(batch=2, n_q_heads=h, n_kv_heads=g, page_size=page, dtype=ck.BF16 if dtype == "bf16" else ck.F32, n_centroids=C, list_len=budget,
                  n_probe=C, top_k=budget)
    idx = ck.ctkvr_build_index(p, tail, [0, C, 2 * C], True, k, table, [budget, budget])
    q = torch.randn((2, h, 128), generator=r).to(base.td)
    sparse, dense = torch.empty((2, h, 128), device=DEV), torch.empty((2, h, 128), dtype=base.td, device=DEV)
    ncand = torch.empty((2, g), dtype=torch.int32, device=DEV)
    ck.ctkvr_decode_step(idx, dev(q), k, v, table, sparse, out_ncand=ncand)
    ck.ctkvr_cache_attn(cache, dev(q), k, v, torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV), kept_dev, table, dense)
    assert (ncand == budget).all()
    st.q, st.k, st.v, st.lens, st.new, st.total = q, k.cpu(), v.cpu(), [budget] * 2, [1, 1], 2
    st.cu, st.cur = torch.tensor([0, 1, 2], dtype=torch.int32), torch.tensor([budget] * 2, dtype=torch.int32)
    want, _, tol, _ = O.attention(st)
    near(dense, want, tol, "dense")
    near(sparse, want, tol, "sparse")
    ck.ctkvr_free(idx)
