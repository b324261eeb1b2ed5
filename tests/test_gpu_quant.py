"""GPU tests of the operators on a paged KV cache of 8-bit rows, in a sliding window and for drafted tokens, against plain 64-bit implementations
(tests/quant_oracle.py): rows appended and read back, attention over them, windows and trees over plain and 8-bit rows, and a run of them together."""
import math
import zlib

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paper_2512_15550_amd as ck
from tests import cache_oracle as O
from tests import quant_oracle as Q
from tests.test_gpu_cache import DEV, HEADS, NAN, SHAPES, cache_of, dev, masks_of, near

STORES = ["int8", "fp8"]
FREQ = 10000.0 ** (-np.arange(64) / 64.0)


def seed_of(*what):
    return zlib.crc32(repr(what).encode()) % 1000


def at(x, *index):
    """x[index] for codes, which torch cannot gather in every type."""
    return x.view(torch.uint8)[index].view(x.dtype) if x.element_size() == 1 else x[index]


def numbers(codes):
    return codes.cpu().float().to(O.F8)


def outputs(st, fill=7.0):
    return torch.full((st.total, st.h, 128), fill, dtype=st.td, device=DEV), torch.full((st.total, st.h), fill, device=DEV)


def pages_of(st):
    return {name: dev(getattr(st, name)) for name in ("k", "k_scales", "v", "v_scales")}


def batch_of(st):
    return dev(st.cu), dev(st.cur), dev(st.table)


def run_quant(st, cache, q=None, **masks):
    out, lse = outputs(st)
    p = pages_of(st)
    ck.ctkvr_cache_quant_attn(cache, dev(st.q) if q is None else q, p["k"], p["k_scales"], p["v"], p["v_scales"], *batch_of(st), out, out_lse=lse,
                              slopes=dev(masks.get("slopes")), prefix_lens=dev(masks.get("prefix")), first_key=dev(masks.get("first")))
    return out, lse


def run_window(st, cache, window, sinks, slopes=None):
    out, lse = outputs(st)
    p = pages_of(st)
    ck.ctkvr_cache_window_attn(cache, dev(st.q), p["k"], p["v"], *batch_of(st), window, out, n_sink=sinks, out_lse=lse, slopes=dev(slopes),
                               k_scales=p["k_scales"], v_scales=p["v_scales"])
    return out, lse


def run_tree(st, cache, mask, first=None):
    out, lse = outputs(st)
    p = pages_of(st)
    ck.ctkvr_cache_tree_attn(cache, dev(st.q), p["k"], p["v"], *batch_of(st), dev(mask), out, out_lse=lse, first_key=dev(first), k_scales=p["k_scales"],
                             v_scales=p["v_scales"])
    return out, lse


def check(st, got, sees, cap=0.0, slopes=None, **more):
    (out, lse), n = got, int(st.cu[-1])
    want, want_lse, tol, tol_lse = Q.attention(st, sees, cap=cap, slopes=slopes, **more)
    near(out[:n], want, tol, "out")
    near(lse[:n], want_lse, tol_lse, "lse")
    assert (out[n:] == 7).all() and (lse[n:] == 7).all(), "tokens behind the last sequence were written"
    return want


def check_quant(st, cap=0.0, slopes=None, prefix=None, first=None):
    check(st, run_quant(st, cache_of(st, softcap=cap), slopes=slopes, prefix=prefix, first=first), lambda b: Q.sees_range(st, b, prefix, first), cap, slopes)


def check_window(st, window, sinks, cap=0.0, slopes=None):
    check(st, run_window(st, cache_of(st, softcap=cap), window, sinks, slopes), lambda b: Q.sees_window(st, b, window, sinks), cap, slopes)


def check_tree(st, mask, cap=0.0, first=None):
    check(st, run_tree(st, cache_of(st, softcap=cap), mask, first), lambda b: Q.sees_tree(st, b, mask, first), cap)


def trees_of(st, branch=3, words=None):
    """A mask for every new token of the batch, of one width; rows behind the last sequence have every bit."""
    words = words or max(1, -(-max(st.new) // 32))
    rows = [Q.tree(n, st.gen, branch, words)[0] for n in st.new if n]
    behind = torch.full((st.total - int(st.cu[-1]), words), -1, dtype=torch.int32)
    return torch.cat(rows + [behind]) if rows else behind


def many(seed, store, dtype, h=32, g=8, page=16, q_scale=1.5):
    """16 sequences with enough new tokens that rows are taken 128 at a time."""
    r = np.random.RandomState(seed)
    lens = [int(x) for x in r.randint(150, 420, size=16)]
    new = [min(s, int(x)) for s, x in zip(lens, r.randint(140, 190, size=16))]
    lens[3], new[3] = 64, 64
    lens[5], new[5] = 300, 1
    lens[7], new[7] = 0, 0
    lens[8], new[8] = 129, 0
    lens[9], new[9] = 400, 400
    return Q.QuantSetup(seed, store, dtype, h, g, page, lens, new, behind=2, q_scale=q_scale)


# ---- append ---------------------------------------------------------------------------------------------------
def run_append(st, store, cache, q, kn, vn, q_out, positions=None):
    """Codes and scales after an append into pages whose bytes and scales were other ones."""
    shape = (st.num_pages, st.g, st.page)
    got = {}
    for name in ("k", "v"):
        got[name] = torch.full(shape + (128,), 0x55, dtype=torch.uint8, device=DEV).view(Q.CODES[store])
        got[name + "_scales"] = torch.full(shape, 9.0, device=DEV)
    ck.ctkvr_cache_quant_append(cache, q, kn, vn, *batch_of(st), q_out, got["k"], got["k_scales"], got["v"], got["v_scales"], positions=dev(positions))
    return got


def places(st):
    """Sequence, slot, page and row in the page of every new token that has one."""
    b = torch.cat([torch.full((m,), i) for i, m in enumerate(st.new)]).long()
    slots = torch.cat([torch.arange(s - m, s) for s, m in zip(st.lens, st.new)])
    return slots, st.table[b, slots // st.page].long(), slots % st.page


def check_rows(store, codes, scales, x, tol, exact):
    """Rows written for x, which a kernel may have off by tol: exact codes where tol is none."""
    want, want_scale, y = Q.quantised(x, store)
    amax = x.abs().amax(dim=-1, keepdim=True).clamp(min=1e-300)
    # (a scale is off by what the largest element is off by, and by the rounding of the quotient)
    assert ((scales.cpu().to(O.F8) - want_scale).abs() <= tol.amax(dim=-1) / Q.TOP[store] + want_scale * 2.0 ** -23).all()
    got = numbers(codes)
    if exact:
        assert torch.equal(got, want)
    # y is off by tol and by the largest element's tol, relative to it, and by roundings of the product and the quotient
    off = (tol + x.abs() / amax * tol.amax(dim=-1, keepdim=True)) / amax * Q.TOP[store] * 1.01 + y.abs() * 2.0 ** -22
    assert ((got - y).abs() <= Q.half_step(y.abs() + off, store) + off).all()


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("axes,given", [(1, False), (1, True), (3, True)])
@pytest.mark.parametrize("h,g,page", [(8, 2, 16), (4, 4, 1), (40, 10, 64)])
def test_append(store, dtype, axes, given, h, g, page):
    st = O.Setup(11, dtype, h, g, page, (40, 1, 0, 130), (17, 1, 0, 65), behind=2)
    axis = np.arange(64) % 3 if axes == 3 else np.zeros(64, int)
    positions = None
    if given:
        positions = torch.randint(-100, 200000, (axes, st.total), generator=st.gen).int()
        positions[:, 0], positions[:, 1], positions[:, 2] = 2 ** 31 - 1, -2 ** 31, 0
    fused = torch.randn((st.total, (h + 2 * g) * 128), generator=st.gen).to(st.td).to(DEV)
    q, kn, vn = (t.view(st.total, -1, 128) for t in torch.split(fused, [h * 128, g * 128, g * 128], dim=1))
    q_out = torch.full((st.total, h, 128), 7.0, dtype=st.td, device=DEV)
    got = run_append(st, store, cache_of(st, rope_axis=axis if axes == 3 else None), q, kn, vn, q_out, positions)
    n = int(st.cu[-1])
    slots, page_of, row = places(st)
    pos = positions[:, :n] if given else slots[None].expand(3, -1)
    want, tol = O.rotated(q[:n].cpu(), pos, FREQ, axis)
    near(q_out[:n], want, tol + want.abs() * O.HALF[dtype], "q")
    assert (q_out[n:] == 7).all()
    wk, tk = O.rotated(kn[:n].cpu(), pos, FREQ, axis)
    spot = page_of.to(DEV), slice(None), row.to(DEV)
    check_rows(store, at(got["k"], *spot), got["k_scales"][spot], wk, tk, False)
    check_rows(store, at(got["v"], *spot), got["v_scales"][spot], vn[:n].cpu().to(O.F8), torch.zeros(vn[:n].shape, dtype=O.F8), dtype == "bf16")
    for name in ("k", "v"):
        got[name].view(torch.uint8)[spot] = 0x55
        got[name + "_scales"][spot] = 9.0
        assert (got[name].view(torch.uint8) == 0x55).all() and (got[name + "_scales"] == 9).all(), "other slots were written"


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_of_rows_that_are_odd(store, dtype):
    """Rows of zeros, of one element, of ties, of the largest and smallest numbers, and with an infinity or NaN: values, and keys at position 0, are held exactly as the
    definition says."""
    big, small = (3.3e38, 1e-37) if dtype == "bf16" else (3.4e38, 1.2e-38)
    rows = torch.randn((14, 1, 128), generator=torch.Generator().manual_seed(1)).to(O.TD[dtype]).float()
    rows[0] = 0.0
    rows[1] = 0.0
    rows[1, 0, 77] = -2.5
    rows[2, 0] = (torch.arange(128) - 64) / 4.0          # 127 / 2 the largest: every other one a tie of int8
    rows[2, 0, 0] = 63.5
    rows[3, 0] = torch.linspace(-448, 448, 128).round()  # e4m3's own range, with its ties
    rows[4] *= big / rows[4].abs().max()
    rows[5] *= small / rows[5].abs().max()
    rows[6, 0, 5] = math.inf
    rows[7, 0, 100] = -math.inf
    rows[8, 0, 0] = NAN
    rows[9, 0, 64] = NAN
    rows[9, 0, 65] = math.inf
    rows[10] = -1.0
    rows[11, 0, ::2] *= 2.0 ** -12                       # the smallest codes of e4m3 and below
    rows[12, 0, :120] *= 2.0 ** -20
    rows[13] *= 2.0 ** 101
    rows = rows.to(O.TD[dtype])
    st = O.Setup(12, dtype, 2, 1, 16, (14,), (14,))
    q = torch.zeros((14, 2, 128), dtype=st.td, device=DEV)
    got = run_append(st, store, cache_of(st), q, dev(rows), dev(rows), q.clone(), torch.zeros((1, 14), dtype=torch.int32))
    slots, page_of, row = places(st)
    want, scale, y = Q.quantised(rows, store)
    odd = torch.isnan(scale[:, 0])
    assert odd.tolist() == [6 <= i <= 9 for i in range(14)]
    for name in ("k", "v"):
        spot = page_of.to(DEV), slice(None), row.to(DEV)
        codes, scales = numbers(at(got[name], *spot)), got[name + "_scales"][spot].cpu().to(O.F8)
        if dtype == "bf16":
            assert torch.equal(codes, want)
        else:     # (24-bit numbers may lie nearer to a border than their quotient's rounding)
            assert ((codes - y).abs() <= Q.half_step(y, store) + y.abs() * 2.0 ** -22).all() and torch.equal(codes[[0, 1, 2, 6, 7, 8, 9, 10]], want[[0, 1, 2, 6, 7, 8, 9, 10]])
        assert torch.isnan(scales[odd]).all() and ((scales - scale)[~odd].abs() <= scale[~odd] * 2.0 ** -23 + 2.0 ** -149).all()


@pytest.mark.parametrize("store", STORES)
def test_append_into_slots_and_pages_that_are_none(store):
    """Tokens beyond the table, before slot 0 and on bad pages are dropped; everything else is written, and nothing else."""
    st = O.Setup(13, "bf16", 4, 2, 16, (64, 30, 40), (10, 30, 5), spare_cols=0)
    st.cur = torch.tensor([68, 20, 40], dtype=torch.int32)     # 4 tokens beyond 64 slots; 10 before slot 0
    st.table[2, 2] = st.num_pages
    kn = torch.randn((45, 2, 128), generator=st.gen).bfloat16().to(DEV)
    got = run_append(st, store, cache_of(st), None, kn, kn, None)
    want = torch.full((st.num_pages, 2, 16, 128), 0x55, dtype=torch.uint8).view(Q.CODES[store])
    codes = Q.quantised(kn.cpu(), store)[0].float().to(Q.CODES[store])
    written = torch.zeros((st.num_pages, 2, 16), dtype=torch.bool)
    for b, (c0, n) in enumerate(((0, 10), (10, 30), (40, 5))):
        for i in range(n):
            slot = int(st.cur[b]) - n + i
            if 0 <= slot < st.cols * 16 and 0 <= int(st.table[b, slot // 16]) < st.num_pages:
                p = int(st.table[b, slot // 16])
                want.view(torch.uint8)[p, :, slot % 16] = codes[c0 + i].view(torch.uint8)
                written[p, :, slot % 16] = True
    assert torch.equal(got["v"].cpu().view(torch.uint8), want.view(torch.uint8))
    for name in ("k", "v"):
        assert torch.equal((got[name].cpu().view(torch.uint8) != 0x55).any(dim=-1), written) and torch.equal((got[name + "_scales"] != 9).cpu(), written)


# ---- reading back ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page,g", [(1, 2), (16, 8), (256, 1)])
@pytest.mark.parametrize("part", ["both", "k", "v"])
def test_read(store, dtype, page, g, part):
    """Every token, or from a first one on (negative, behind the end), with pages that are none on either side and an out_table narrower than the rows."""
    st = Q.QuantSetup(seed_of(store, dtype, page), store, dtype, 2 * g, g, page, (300, 1, 0, 70, 515), (0,) * 5)
    if page < 256:
        st.table[0, 3], st.table[3, 0] = -1, st.num_pages
    cache = cache_of(st)
    for first, cols in ((None, st.cols), (None, max(1, 64 // page)), ((0, -5, 3, 69, 200), st.cols), ((37, 0, 0, 2 ** 31 - 1, 515), st.cols)):
        pool = st.batch * cols + 2
        out_table = torch.randperm(pool, generator=st.gen)[:st.batch * cols].view(st.batch, cols).int()
        if cols > 2:
            out_table[0, 1], out_table[4, 2] = -7, pool
        pages = [torch.full((pool, g, page, 128), 5.0, dtype=st.td, device=DEV) for _ in range(2)]
        want = [x.cpu().clone() for x in pages]
        p = pages_of(st)
        drop = {"both": (), "k": (2, 3), "v": (0, 1)}[part]
        rows = [None if i in drop else x for i, x in enumerate((p["k"], p["k_scales"], p["v"], p["v_scales"]))]
        ck.ctkvr_cache_quant_read(cache, *rows, dev(st.cur), dev(st.table), dev(out_table), pages[0] if part != "v" else None, pages[1] if part != "k" else None,
                                  first_tokens=None if first is None else dev(torch.tensor(first, dtype=torch.int32)))
        for i, name in enumerate(("k", "v")):
            if part not in ("both", name):
                continue
            values = (getattr(st, name).float() * getattr(st, name + "_scales")[..., None]).to(st.td)     # one product in fp32, one rounding
            for b, s in enumerate(st.lens):
                f = 0 if first is None else max(0, first[b])
                for j in range(max(0, min(s - f, cols * page))):
                    src, dst = int(st.table[b, (f + j) // page]), int(out_table[b, j // page])
                    if 0 <= src < st.num_pages and 0 <= dst < pool:
                        want[i][dst, :, j % page] = values[src, :, (f + j) % page]
        assert all(torch.equal(a.cpu(), w) for a, w in zip(pages, want))


def test_read_of_more_tokens_than_blocks_take_at_once():
    st = Q.QuantSetup(15, "int8", "bf16", 8, 8, 64, (9000, 20000), (0, 0))
    pages = [torch.zeros((st.num_pages, 8, 64, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    p = pages_of(st)
    ck.ctkvr_cache_quant_read(cache_of(st), p["k"], p["k_scales"], p["v"], p["v_scales"], dev(st.cur), dev(st.table), dev(st.table), *pages)
    for got, name in zip(pages, ("k", "v")):
        want = (getattr(st, name).float() * getattr(st, name + "_scales")[..., None]).bfloat16()
        for b, s in enumerate(st.lens):
            t = torch.arange(s)
            page = st.table[b, t // 64].long()
            assert torch.equal(got.cpu()[page, :, t % 64], want[page, :, t % 64])


# ---- attention over 8-bit rows ------------------------------------------------------------------------------------
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h,g", HEADS)
def test_attention(shape, store, dtype, h, g):
    lens, new = SHAPES[shape]
    check_quant(Q.QuantSetup(seed_of(shape, dtype, h, store), store, dtype, h, g, 16, lens, new, q_scale=2.0))


@pytest.mark.parametrize("kinds", [("bias",), ("prefix",), ("docs",), ("window", "bias"), ("bias", "prefix", "docs")], ids="+".join)
@pytest.mark.parametrize("cap", [0.0, 5.0])
@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", ["few", "many"])
def test_masks_cap_and_bias(kinds, cap, store, dtype, shape):
    if shape == "many":
        st = many(51 + len(kinds), store, dtype, h=16, g=4)
    else:
        st = Q.QuantSetup(len(kinds) * 10 + int(cap), store, dtype, 8, 2, 16, (330, 77, 150), (200, 1, 150), behind=3, q_scale=2.0)
    check_quant(st, cap=cap, **masks_of(st, kinds))


@pytest.mark.parametrize("page", [1, 2, 64, 256])
@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("new", [(71, 33), (1, 1)])
def test_page_sizes(page, store, new):
    check_quant(Q.QuantSetup(page, store, "bf16", 8, 2, page, (page + 70, 200), new))


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("page", [1, 16, 64])
def test_many_rows_and_pages_that_are_none(store, page):
    st = many(60 + page, store, "bf16", page=page)
    for b in (0, 4, 9):
        for i, c in enumerate([c for c in (0, 1, 5, 70, 71) if c < -(-st.lens[b] // page)][:3]):
            st.table[b, c] = (st.num_pages, -1, -2 ** 31)[i]
    check_quant(st)
    st = Q.QuantSetup(4, store, "f32", 8, 2, page, (200, 900, 33), (60, 1, 33))
    for b, cols in ((0, (0, 3, 4, 5, 6, 11)), (1, (7, 13)), (2, (0,))):
        for c in cols:
            if c < st.cols:
                st.table[b, c] = st.num_pages
    check_quant(st)


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_see_nothing(store, dtype):
    st = Q.QuantSetup(3, store, dtype, 4, 1, 16, (90, 40), (90, 5))
    first = torch.zeros(st.total, dtype=torch.int32)
    first[10:20] = 50
    first[70] = 2 ** 31 - 1
    st.table[1] = -1
    check_quant(st, first=first)
    out, lse = run_quant(st, cache_of(st), first=first)
    for rows in (slice(10, 20), slice(70, 71), slice(90, 95)):
        assert not out[rows].any() and (lse[rows] == -math.inf).all()


def spoil(st, pages, rows):
    """Every byte a NaN of e4m3 and every scale one, in these rows of these pages (the others' of plain rows: NaN)."""
    for name in ("k", "v"):
        if st.store == "plain":
            getattr(st, name)[pages, :, rows] = NAN
        else:
            getattr(st, name).view(torch.uint8)[pages, :, rows] = 0xff
            getattr(st, name + "_scales")[pages, :, rows] = NAN


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", ["few", "many"])
def test_what_is_not_seen_does_not_matter(store, dtype, shape):
    """Bytes that nobody wrote behind the last key of a page, on pages that are free, and rows of NaN that are hidden by position or by a document."""
    if shape == "many":
        st = many(71, store, dtype, h=8, g=8)
    else:
        st = Q.QuantSetup(5, store, dtype, 8, 2, 32, (150, 71), (100, 71))
    first, hidden = torch.zeros(st.total, dtype=torch.int32), []
    for b, (s, n) in enumerate(zip(st.lens, st.new)):
        if s % st.page:
            spoil(st, int(st.table[b, (s - 1) // st.page]), slice(s % st.page, st.page))
        if n > 20:                      # one token's row: the earlier ones do not see it, and the later ones' documents begin behind it
            t, i = s - n // 2, int(st.cu[b]) + n - n // 2
            spoil(st, int(st.table[b, t // st.page]), t % st.page)
            first[i + 1:int(st.cu[b + 1])] = t + 1
            hidden.append(i)
    spoil(st, sorted(set(range(st.num_pages)) - set(st.table[st.table >= 0].tolist())), slice(None))
    out, lse = run_quant(st, cache_of(st), first=first)
    keep = [i for i in range(int(st.cu[-1])) if i not in hidden]
    clean = lambda b: Q.sees_range(st, b, first=first) & ~torch.isin(torch.arange(st.lens[b]), torch.tensor([st.lens[b] - st.new[b] // 2]))  # noqa: E731
    want, want_lse, tol, tol_lse = Q.attention(st, lambda b: clean(b) if st.new[b] > 20 else Q.sees_range(st, b, first=first))
    near(out[keep], want[keep], tol[keep], "out")
    near(lse[keep], want_lse[keep], tol_lse[keep], "lse")


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_row_of_nan_that_is_seen(store, dtype):
    """A value whose row is NaN makes the rows that see it NaN, and no others; a key's makes their sums NaN."""
    st = Q.QuantSetup(6, store, dtype, 4, 2, 16, (100,), (100,))
    page = int(st.table[0, 40 // 16])
    st.v_scales[page, 1, 40 % 16] = NAN
    st.v[page, 1, 40 % 16] = 0
    out, lse = run_quant(st, cache_of(st))
    assert torch.isfinite(lse).all() and torch.isfinite(out[:40]).all() and torch.isfinite(out[:, :2]).all() and torch.isnan(out[40:, 2:]).all()
    st.k_scales[page, 0, 40 % 16] = NAN
    out, lse = run_quant(st, cache_of(st))
    assert torch.isfinite(lse[:40]).all() and torch.isfinite(lse[:, 2:]).all() and torch.isnan(lse[40:, :2]).all() and torch.isfinite(out[:40]).all()


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("dtype,lens,new,h,g", [("bf16", (4300, 5000), (140, 131), 8, 1), ("bf16", (6000,), (70,), 16, 2), ("f32", (3000,), (1,), 4, 1),
                                                ("bf16", (9000, 300), (1, 1), 8, 2), ("f32", (2500, 40), (30, 3), 8, 2)])
def test_keys_split(store, dtype, lens, new, h, g):
    st = Q.QuantSetup(81, store, dtype, h, g, 16, lens, new, q_scale=2.0)
    check_quant(st, cap=5.0, **masks_of(st, ("prefix", "bias")))
    check_quant(st, **masks_of(st, ("window",)))


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("powers", [3, 12, 60])
@pytest.mark.parametrize("shape", ["few", "split", "many"])
def test_values_of_very_different_sizes(store, dtype, powers, shape):
    """Rows of values apart by up to 2^120, in any order, some of them zeros; bytes on free pages that would be larger still."""
    if shape == "many":
        st = many(83, store, dtype, h=16, g=4)
    else:
        st = Q.QuantSetup(83, store, dtype, 8, 2, 16, (2500, 40, 600) if shape == "split" else (150, 64, 1), (1, 3, 2) if shape == "split" else (100, 1, 1), q_scale=2.0)
    by = torch.randint(-powers, powers + 1, st.v_scales.shape, generator=st.gen)
    st.v_scales = st.v_scales * torch.exp2(by.float())
    zero = torch.rand(st.v_scales.shape, generator=st.gen) < 0.05
    st.v_scales[zero] = 0.0
    st.v.view(torch.uint8)[zero] = 0
    free = sorted(set(range(st.num_pages)) - set(st.table[st.table >= 0].tolist()))
    st.v_scales[free] = 1e38
    for b, s in enumerate(st.lens):
        if s % st.page:
            st.v_scales[int(st.table[b, (s - 1) // st.page]), :, s % st.page:] = 1e38
    check(st, run_quant(st, cache_of(st)), lambda b: Q.sees_range(st, b), spread=True)


LARGE = {
    "few": ((90, 300, 64), (16, 4, 1)),
    "drafts": ((90, 300), (40, 33)),
    "split": ((6000,), (3,)),
    "rows": ((400, 2000), (400, 150)),
    "rows_split": ((6000,), (150,)),
}


@pytest.mark.parametrize("kind", ["quant", "docs", "window", "tree"])
@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", LARGE)
@pytest.mark.parametrize("power,others", [(30, 0), (110, 0), (190, -70)])
def test_large_values_that_other_tokens_see(kind, store, dtype, shape, power, others):
    """Values up to 2^190 times as large as the others (times 2^`others`), which some tokens see and their neighbours do not: these are as exact as without them."""
    lens, new = LARGE[shape]
    st = Q.QuantSetup(seed_of(kind, store, dtype, shape), store, dtype, 16, 2, 16, lens, new, behind=1, q_scale=2.0)
    n, first, mask = int(st.cu[-1]), None, trees_of(st)
    sees = {"quant": lambda b: Q.sees_range(st, b), "docs": lambda b: Q.sees_range(st, b, None, first), "window": lambda b: Q.sees_window(st, b, 70, 3),
            "tree": lambda b: Q.sees_tree(st, b, mask)}[kind]
    if kind == "docs":
        first = torch.randint(0, 2, (st.total,), generator=st.gen).int() * 45
    large = []
    st.v_scales *= 2.0 ** others
    for b, (s, m) in enumerate(zip(lens, new)):
        large.append({"docs": 31, "window": max(s - m - 40, 0)}.get(kind, s - m // 2 - 1))     # before the others' first key, in some windows, half of the new tokens on
        for part in (power // 2, power - power // 2):     # (2^190 is no fp32 number)
            st.v_scales[int(st.table[b, large[b] // 16]), :, large[b] % 16] *= 2.0 ** part
    assert torch.isfinite(st.v_scales).all()
    if kind == "quant":
        got = run_quant(st, cache_of(st))
    elif kind == "docs":
        got = run_quant(st, cache_of(st), first=first)
    elif kind == "window":
        got = run_window(st, cache_of(st), 70, 3)
    else:
        got = run_tree(st, cache_of(st), mask)
    out, lse = (x[:n].cpu() for x in got)
    hit = torch.cat([sees(b)[:, large[b]] for b in range(st.batch)])
    want, want_lse, tol, tol_lse = Q.attention(st, sees, spread=True)
    near(out[hit], want[hit], tol[hit], "tokens that see it")
    near(lse, want_lse, tol_lse, "lse")
    for b in range(st.batch):
        st.v_scales[int(st.table[b, large[b] // 16]), :, large[b] % 16] = 1.0
    want, _, tol, _ = Q.attention(st, sees)
    assert (~hit).any() or shape in ("few", "split")
    near(out[~hit], want[~hit], tol[~hit], "tokens that do not")


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_views_of_a_fused_projection_and_a_scale_of_ones_own(store, dtype):
    st = Q.QuantSetup(7, store, dtype, 8, 2, 16, (70, 90), (70, 40))
    fused = torch.full((st.total, 12 * 128 + 64), NAN, dtype=st.td, device=DEV)
    q = fused[:, :8 * 128].view(st.total, 8, 128)
    q.copy_(st.q)
    cache = cache_of(st, sm_scale=0.25)
    a, b = run_quant(st, cache, q=q), run_quant(st, cache)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    check(st, a, lambda b: Q.sees_range(st, b), scale=0.25)


@pytest.mark.parametrize("store", STORES)
def test_a_cache_beyond_32_bit_offsets(store):
    """Rows whose byte offsets pass 2^32: attention, a window, a tree, append and read."""
    g, page, pool = 8, 16, 280000                   # 2^32 bytes are 262144 pages
    st = Q.QuantSetup(9, store, "bf16", 8, g, page, (100,), (30,))
    used = st.table[0, :7].long()
    far = (pool - 1 - used).to(DEV)
    big = {}
    for name in ("k", "v"):
        big[name] = torch.empty((pool, g, page, 128), dtype=torch.uint8, device=DEV)
        big[name][far] = getattr(st, name).view(torch.uint8)[used].to(DEV)
        big[name] = big[name].view(Q.CODES[store])
        big[name + "_scales"] = torch.empty((pool, g, page), device=DEV)
        big[name + "_scales"][far] = getattr(st, name + "_scales")[used].to(DEV)
    table = torch.where(st.table >= 0, pool - 1 - st.table, -1).to(DEV)
    cache, batch = cache_of(st, num_pages=pool), (dev(st.cu), dev(st.cur), table)
    codes = [big[x] for x in ("k", "k_scales", "v", "v_scales")]
    out, lse = outputs(st)
    ck.ctkvr_cache_quant_attn(cache, dev(st.q), *codes, *batch, out, out_lse=lse)
    check(st, (out, lse), lambda b: Q.sees_range(st, b))
    ck.ctkvr_cache_window_attn(cache, dev(st.q), big["k"], big["v"], *batch, 20, out, n_sink=3, out_lse=lse, k_scales=big["k_scales"], v_scales=big["v_scales"])
    check(st, (out, lse), lambda b: Q.sees_window(st, b, 20, 3))
    kn = torch.randn((30, g, 128), generator=st.gen).bfloat16().to(DEV)
    ck.ctkvr_cache_quant_append(cache, None, kn, kn, *batch, None, *codes)
    pages = torch.zeros((10, g, page, 128), dtype=torch.bfloat16, device=DEV)
    ck.ctkvr_cache_quant_read(cache, None, None, big["v"], big["v_scales"], dev(st.cur), table, torch.arange(7, dtype=torch.int32, device=DEV)[None].contiguous(),
                              None, pages)
    c, s, _ = Q.quantised(kn.cpu(), store)
    t = torch.arange(70, 100)
    # (a value off by its scale's rounding and its own)
    near(pages[t // 16, :, t % 16], c * s[..., None], (c * s[..., None]).abs() * (2.0 ** -8 + 2.0 ** -22), "values")


# ---- windows --------------------------------------------------------------------------------------------------
ALL_STORES = ["plain"] + STORES


@pytest.mark.parametrize("store", ALL_STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 4), (32, 0), (33, 33), (64, 64), (65, 4), (100, 70), (64, 10 ** 6), (10 ** 9, 0), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_windows(store, dtype, window, sinks):
    st = Q.QuantSetup(seed_of(store, window), store, dtype, 8, 2, 16, (330, 77, 700, 1, 0), (200, 1, 1, 1, 0), behind=3, q_scale=2.0)
    check_window(st, window, sinks)


@pytest.mark.parametrize("store", ALL_STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap", [0.0, 4.0])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("shape", ["tokens", "many", "split"])
def test_windows_with_cap_and_bias(store, dtype, cap, bias, shape):
    if shape == "many":
        st = many(61, store, dtype, h=16, g=4)
    elif shape == "split":
        st = Q.QuantSetup(62, store, dtype, 8, 1, 16, (6000,), (70 if dtype == "bf16" else 9,), q_scale=2.0)
    else:
        st = Q.QuantSetup(63, store, dtype, 16, 2, 16, (900, 2000, 64, 30), (1, 1, 1, 1), q_scale=2.0)
    slopes = masks_of(st, ("bias",))["slopes"] if bias else None
    for window, sinks in ((50, 4), (130, 0), (3000, 40)):
        check_window(st, window, sinks, cap, slopes)


@pytest.mark.parametrize("store", ALL_STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 40, 300])
def test_pages_before_a_window_are_not_needed(store, dtype, new):
    """Pages between the first tokens and the window: none (-1), or another sequence's with bytes that nobody wrote."""
    st = Q.QuantSetup(64, store, dtype, 8, 2, 16, (900, 700), (new, new), q_scale=2.0)
    window, sinks = 100, 20
    cache = cache_of(st)
    want = run_window(st, cache, window, sinks)
    check(st, want, lambda b: Q.sees_window(st, b, window, sinks))
    free = sorted(set(range(st.num_pages)) - set(st.table[st.table >= 0].tolist()))
    spoil(st, free, slice(None))
    for b, s in enumerate(st.lens):
        gone = range(-(-sinks // 16), (s - new + 1 - window) // 16)      # whole pages behind the first tokens and before the earliest window
        for i, c in enumerate(gone):
            spoil(st, int(st.table[b, c]), slice(None))
            st.table[b, c] = -1 if i % 2 else free[i % len(free)]
    got = run_window(st, cache, window, sinks)
    check(st, got, lambda b: Q.sees_window(st, b, window, sinks))


@pytest.mark.parametrize("store", ALL_STORES)
def test_windows_of_pages_of_one_and_with_no_pages(store):
    st = Q.QuantSetup(65, store, "bf16", 8, 2, 1, (200, 129), (60, 1), q_scale=2.0)
    for c in (0, 2, 150, 199):
        st.table[0, c] = -1
    check_window(st, 40, 3)
    st.table[:] = -1
    out, lse = run_window(st, cache_of(st), 40, 3)
    assert not out.any() and (lse == -math.inf).all()


# ---- trees ----------------------------------------------------------------------------------------------------
TREES = {
    "one": ((1, 40), (1, 1)),
    "drafts": ((300, 64, 129, 20), (17, 5, 33, 20)),
    "edges": ((95, 96, 97, 64, 65, 128), (31, 32, 33, 64, 1, 63)),
    "wide": ((700, 100), (200, 100)),
    "long": ((5000,), (40,)),
    "none": ((50, 0, 130), (0, 0, 130)),
}


@pytest.mark.parametrize("shape", TREES)
@pytest.mark.parametrize("store", ALL_STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h,g", [(4, 4), (8, 2), (16, 2)])
def test_trees(shape, store, dtype, h, g):
    lens, new = TREES[shape]
    st = Q.QuantSetup(seed_of(shape, dtype, h, store), store, dtype, h, g, 16, lens, new, behind=2, q_scale=2.0)
    check_tree(st, trees_of(st))


@pytest.mark.parametrize("store", ALL_STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap", [0.0, 4.0])
@pytest.mark.parametrize("shape", ["few", "many"])
def test_masks_that_are_no_trees(store, dtype, cap, shape):
    """Any bits: later tokens, not the token itself, none at all, beyond the sequence's tokens; a first key besides."""
    if shape == "many":
        st = many(66, store, dtype, h=16, g=4)
    else:
        st = Q.QuantSetup(67, store, dtype, 8, 2, 32, (90, 300, 25), (50, 70, 25), behind=2, q_scale=2.0)
    words = -(-max(st.new) // 32) + 1
    mask = torch.randint(-2 ** 31, 2 ** 31, (st.total, words), generator=st.gen).int()
    mask[3:9] = 0
    mask[11] = -1
    check_tree(st, mask, cap)
    first = torch.randint(-10, 200, (st.total,), generator=st.gen).int()
    first[5] = 2 ** 31 - 1
    check_tree(st, mask, cap, first)
    check_tree(st, mask[:, :1].contiguous(), cap)       # fewer bits than tokens: the others are not seen


@pytest.mark.parametrize("store", ALL_STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_trees_without_anything_to_see(store, dtype):
    st = Q.QuantSetup(68, store, dtype, 8, 2, 16, (9, 30), (9, 4), q_scale=2.0)
    mask = trees_of(st)
    mask[2] = 0
    mask[5] = 1 << 20
    out, lse = run_tree(st, cache_of(st), mask)
    assert not out[2].any() and not out[5].any() and (lse[2] == -math.inf).all() and (lse[5] == -math.inf).all()
    check_tree(st, mask)


@pytest.mark.parametrize("store", ALL_STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_drafted_tokens_of_other_branches_do_not_matter(store, dtype):
    """A drafted token whose row is NaN: only those that see it are."""
    st = Q.QuantSetup(69, store, dtype, 8, 2, 16, (200,), (20,), q_scale=2.0)
    mask = trees_of(st)
    bad = 6
    spoil(st, int(st.table[0, 186 // 16]), 186 % 16)
    out, lse = run_tree(st, cache_of(st), mask)
    sees = (mask[:, 0] >> bad & 1).bool()
    assert sees.any() and not sees.all()
    assert torch.isnan(out[sees.to(DEV)]).all() and torch.isfinite(out[~sees.to(DEV)]).all()
    want, want_lse, tol, tol_lse = Q.attention(st, lambda b: Q.sees_tree(st, b, torch.where(sees[:, None], 0, mask)))
    near(out.cpu()[~sees], want[~sees], tol[~sees], "out")
    near(lse.cpu()[~sees], want_lse[~sees], tol_lse[~sees], "lse")


@pytest.mark.parametrize("store", ALL_STORES)
def test_trees_on_pages_that_are_none_and_beyond_the_table(store):
    st = Q.QuantSetup(70, store, "bf16", 8, 2, 16, (200, 64), (40, 10), spare_cols=0)
    st.table[0, 4], st.table[0, 11] = -1, st.num_pages
    check_tree(st, trees_of(st))
    st.cur = torch.tensor([208, 70], dtype=torch.int32)     # tokens beyond the table's slots are no keys; those that they belong to attend all the same
    mask = trees_of(st)
    out, lse = run_tree(st, cache_of(st), mask)
    st.lens = [208, 64]

    def sees(b):
        if b == 0:
            return Q.sees_tree(st, 0, mask)
        seen = torch.zeros((10, 64), dtype=torch.bool)
        seen[:, :60] = True
        bits = mask[40:50, 0].long()
        for j in range(4):
            seen[:, 60 + j] = (bits >> j & 1).bool()
        return seen
    check(st, (out, lse), sees)


# ---- many rows in wide tables ---------------------------------------------------------------------------------
def wide(seed, store, page, lens=(300, 200, 700, 64), new=(100, 70, 129, 64), h=8, g=2, **more):
    """Tables with room for more than 4096 tokens: rows are taken 256 at a time."""
    return Q.QuantSetup(seed, store, "bf16", h, g, page, lens, new, spare_cols=4096 // page, behind=2, **more)


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("page", [1, 8, 64])
@pytest.mark.parametrize("cap", [0.0, 5.0])
@pytest.mark.parametrize("kinds", [(), ("bias",), ("prefix",), ("docs",), ("bias", "prefix", "docs")], ids="+".join)
def test_wide_tables(store, page, cap, kinds):
    st = wide(seed_of(store, page, kinds), store, page, q_scale=2.0)
    check_quant(st, cap=cap, **masks_of(st, kinds))


@pytest.mark.parametrize("store", ALL_STORES)
@pytest.mark.parametrize("page", [1, 4, 8, 64])
@pytest.mark.parametrize("cap", [0.0, 5.0])
def test_wide_tables_of_drafts(store, page, cap):
    """Any bits, a first key besides; pages that are none."""
    st = wide(seed_of(store, page), store, page, q_scale=2.0)
    mask = torch.randint(-2 ** 31, 2 ** 31, (st.total, 5), generator=st.gen).int()
    mask[3:9] = 0
    first = torch.randint(-10, 200, (st.total,), generator=st.gen).int()
    check_tree(st, mask, cap)
    check_tree(st, mask, cap, first)
    for b, c in ((0, 1), (0, 100 // page), (1, 0), (2, 650 // page), (3, 63 // page)):
        st.table[b, c] = st.num_pages if b % 2 else -1
    check_tree(st, mask, cap, first)


@pytest.mark.parametrize("store", ALL_STORES)
@pytest.mark.parametrize("page", [1, 8, 16])
def test_wide_tables_what_is_not_seen_does_not_matter(store, page):
    """A drafted token's row of NaN, for those that do not see it; bytes that nobody wrote behind the last key and on pages that are free."""
    st = wide(seed_of(store, page), store, page, q_scale=2.0)
    mask, bad = trees_of(st), 20
    spoil(st, sorted(set(range(st.num_pages)) - set(st.table[st.table >= 0].tolist())), slice(None))
    sees = torch.zeros(int(st.cu[-1]), dtype=torch.bool)
    for b, (s, n) in enumerate(zip(st.lens, st.new)):
        if s % page:
            spoil(st, int(st.table[b, (s - 1) // page]), slice(s % page, page))
        t = s - n + bad
        spoil(st, int(st.table[b, t // page]), t % page)
        rows = slice(int(st.cu[b]), int(st.cu[b + 1]))
        sees[rows] = (mask[rows, 0] >> bad & 1).bool()
    out, lse = run_tree(st, cache_of(st), mask)
    want, want_lse, tol, tol_lse = Q.attention(st, lambda b: Q.sees_tree(st, b, torch.where((mask[:, 0] >> bad & 1).bool()[:, None], 0, mask)))
    n = int(st.cu[-1])
    assert torch.isnan(out[:n][sees.to(DEV)]).all()
    near(out[:n].cpu()[~sees], want[~sees], tol[~sees], "out")
    near(lse[:n].cpu()[~sees], want_lse[~sees], tol_lse[~sees], "lse")
    assert (out[n:] == 7).all() and (lse[n:] == 7).all()


@pytest.mark.parametrize("store", ALL_STORES)
@pytest.mark.parametrize("page", [1, 8, 16])
@pytest.mark.parametrize("sinks", [0, 100])
def test_wide_tables_of_windows(store, page, sinks):
    st = wide(seed_of(store, page, sinks), store, page, (4500, 4300), (150, 129), q_scale=2.0)
    check_window(st, 4100, sinks)
    check_window(st, 4097, sinks, cap=5.0, slopes=masks_of(st, ("bias",))["slopes"])


# ---- calls of every kind --------------------------------------------------------------------------------------
KINDS = [("quant", "int8"), ("quant", "fp8")] + [(kind, store) for kind in ("window", "tree") for store in ALL_STORES]


def check_kind(st, kind, window=60, sinks=5):
    if kind == "quant":
        check_quant(st)
    elif kind == "window":
        check_window(st, window, sinks)
    else:
        check_tree(st, trees_of(st))


@pytest.mark.parametrize("kind,store", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch", [65, 130])
def test_more_sequences_than_a_wave_has_lanes(kind, store, dtype, batch):
    """Blocks look their sequence up 64 at a time: sequences without new tokens, single tokens, drafts and a chunk on either side of the 64th."""
    r = np.random.RandomState(batch)
    new = [int(x) for x in r.choice([0, 1, 1, 1, 2, 7], size=batch)]
    new[62:66] = [0, 5, 40, 0][:len(new[62:66])]
    lens = [int(x) + n for x, n in zip(r.randint(0, 120, size=batch), new)]
    check_kind(Q.QuantSetup(seed_of(kind, store, dtype, batch), store, dtype, 4, 1, 16, lens, new, behind=3, q_scale=2.0), kind)


@pytest.mark.parametrize("kind,store", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_prompt_s_chunk_beside_single_tokens(kind, store, dtype):
    st = Q.QuantSetup(seed_of(kind, store, dtype), store, dtype, 8, 2, 16, (90, 600, 33, 1, 257, 512), (1, 400, 1, 1, 1, 2), behind=1, q_scale=2.0)
    check_kind(st, kind)


@pytest.mark.parametrize("kind,store", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [(1, 1, 1), (130, 1, 64)])
def test_sequences_that_share_their_first_pages(kind, store, dtype, new):
    st = Q.QuantSetup(seed_of(kind, store, dtype, new), store, dtype, 8, 2, 16, (300, 200, 250), new, q_scale=2.0)
    st.table[1, :4] = st.table[2, :4] = st.table[0, :4]
    check_kind(st, kind, window=100)


@pytest.mark.parametrize("kind,store", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [(1, 1, 1), (20, 1, 3), (150, 40, 1)])
def test_a_query_that_is_not_finite_is_its_own_row_s_trouble(kind, store, dtype, new):
    """A head's query of NaN, another's with an infinity, and NaN behind the last sequence."""
    st = Q.QuantSetup(seed_of(kind, store, dtype), store, dtype, 8, 2, 16, (300, 200, 250), new, behind=4, q_scale=2.0)
    n = int(st.cu[-1])
    st.q[n:] = NAN
    whole = st.q.clone()
    st.q[0, 3] = NAN
    st.q[n - 1, 6, 77] = math.inf
    run = {"quant": lambda: run_quant(st, cache_of(st)), "window": lambda: run_window(st, cache_of(st), 60, 5), "tree": lambda: run_tree(st, cache_of(st), mask)}[kind]
    mask = trees_of(st)
    out, lse = run()
    st.q = whole
    sees = {"quant": lambda b: Q.sees_range(st, b), "window": lambda b: Q.sees_window(st, b, 60, 5), "tree": lambda b: Q.sees_tree(st, b, mask)}[kind]
    want, want_lse, tol, tol_lse = Q.attention(st, sees)
    fine = torch.ones((n, 8), dtype=torch.bool)
    fine[0, 3] = fine[n - 1, 6] = False
    near(out[:n].cpu()[fine], want[fine], tol[fine], "out")
    near(lse[:n].cpu()[fine], want_lse[fine], tol_lse[fine], "lse")
    assert torch.isnan(out[0, 3]).all() and (out[n:] == 7).all() and (lse[n:] == 7).all()


@pytest.mark.parametrize("kind,store", KINDS)
@pytest.mark.parametrize("new", [(1, 1), (33, 2)])
def test_without_log_sums_and_without_tokens(kind, store, new):
    """The same outputs where no log-sum-exp is wanted; a call of no tokens writes nothing."""
    st = Q.QuantSetup(seed_of(kind, store), store, "bf16", 8, 2, 16, (3000, 70), new, q_scale=2.0)
    cache, p, mask, q = cache_of(st), pages_of(st), dev(trees_of(st)), dev(st.q)

    def call(cu, q, out, lse, mask):
        batch = (cu,) + batch_of(st)[1:]
        if kind == "quant":
            ck.ctkvr_cache_quant_attn(cache, q, p["k"], p["k_scales"], p["v"], p["v_scales"], *batch, out, out_lse=lse)
        elif kind == "window":
            ck.ctkvr_cache_window_attn(cache, q, p["k"], p["v"], *batch, 1000, out, n_sink=5, out_lse=lse, k_scales=p["k_scales"], v_scales=p["v_scales"])
        else:
            ck.ctkvr_cache_tree_attn(cache, q, p["k"], p["v"], *batch, mask, out, out_lse=lse, k_scales=p["k_scales"], v_scales=p["v_scales"])

    out, lse = outputs(st)
    call(dev(st.cu), q, out, lse, mask)
    alone = torch.full_like(out, 7.0)
    call(dev(st.cu), q, alone, None, mask)
    assert torch.equal(out, alone)
    kept = out.clone()
    call(torch.zeros_like(dev(st.cu)), q[:0], out[:0], lse[:0], mask[:0])
    call(torch.zeros_like(dev(st.cu)), q, out, lse, mask)
    assert torch.equal(out, kept)


@pytest.mark.parametrize("store", ALL_STORES)
@pytest.mark.parametrize("new", [(40, 10), (300, 4)])
def test_windows_beyond_the_table(store, new):
    """Tokens beyond the table's slots are no keys; they attend all the same, in a window that ends behind the last key."""
    st = Q.QuantSetup(seed_of(store, new), store, "bf16", 8, 2, 16, (320, 64), new, spare_cols=0)
    st.cur = torch.tensor([320 + 30, 64 + 6], dtype=torch.int32)
    got = run_window(st, cache_of(st), 50, 3)
    st.lens = [320, 70]

    def sees(b):
        cur = int(st.cur[b])
        pos, t = torch.arange(cur - new[b], cur)[:, None], torch.arange(st.lens[b])[None, :]
        return (t <= pos) & ((t > pos - 50) | (t < 3))
    check(st, got, sees)


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h,g,tokens", [(32, 8, 5), (8, 2, 700)])
def test_append_rotates_queries_in_place(store, dtype, h, g, tokens):
    st = O.Setup(14, dtype, h, g, 16, (tokens + 20,), (tokens,))
    q, kn, vn = (torch.randn((tokens, n, 128), generator=st.gen).to(st.td).to(DEV) for n in (h, g, g))
    there = q.clone()
    want_q, cache = torch.empty_like(q), cache_of(st)
    want = run_append(st, store, cache, q, kn, vn, want_q)
    got = run_append(st, store, cache, there, kn, vn, there)
    assert torch.equal(there, want_q)
    assert all(torch.equal(got[name].view(torch.uint8), want[name].view(torch.uint8)) for name in ("k", "v"))


# ---- streams, graphs, repetition ------------------------------------------------------------------------------
@pytest.mark.parametrize("kind,store", KINDS)
def test_two_handles_on_two_streams_at_once(kind, store):
    """Split calls, each with a workspace of its own, that run beside each other."""
    sts = [Q.QuantSetup(seed, store, "bf16", 8, 2, 16, (6000, 5000), new, q_scale=2.0) for seed, new in ((81, (1, 2)), (82, (60, 40)))]
    calls = []
    for st in sts:
        cache, p, batch, q, mask = cache_of(st), pages_of(st), batch_of(st), dev(st.q), dev(trees_of(st))

        def call(out, lse, cache=cache, p=p, batch=batch, q=q, mask=mask):
            if kind == "quant":
                ck.ctkvr_cache_quant_attn(cache, q, p["k"], p["k_scales"], p["v"], p["v_scales"], *batch, out, out_lse=lse)
            elif kind == "window":
                ck.ctkvr_cache_window_attn(cache, q, p["k"], p["v"], *batch, 4500, out, n_sink=5, out_lse=lse, k_scales=p["k_scales"], v_scales=p["v_scales"])
            else:
                ck.ctkvr_cache_tree_attn(cache, q, p["k"], p["v"], *batch, mask, out, out_lse=lse, k_scales=p["k_scales"], v_scales=p["v_scales"])
        calls.append(call)
    alone, beside = [outputs(st) for st in sts], [outputs(st) for st in sts]
    for call, outs in zip(calls, alone):
        call(*outs)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sts]
    for _ in range(5):
        for stream, call, outs in zip(streams, calls, beside):
            with torch.cuda.stream(stream):
                call(*outs)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for x, y in zip(alone, beside) for a, b in zip(x, y))


@pytest.mark.parametrize("kind,store", [("quant", "int8"), ("quant", "fp8")] + [(kind, store) for kind in ("window", "tree") for store in ALL_STORES])
@pytest.mark.parametrize("new", [1, 33])
def test_the_same_call_gives_the_same_bits_on_any_stream_and_in_graphs(kind, store, new):
    """Eagerly, on another stream, and in two graphs on one handle that take turns, with eager work between."""
    st = Q.QuantSetup(31, store, "bf16", 4, 1, 16, (3000,) if new == 1 else (3000, 700), (new,) if new == 1 else (new, new), q_scale=2.0)
    cache, p, batch, q, mask = cache_of(st), pages_of(st), batch_of(st), dev(st.q), dev(trees_of(st))

    def call(out, lse):
        if kind == "quant":
            ck.ctkvr_cache_quant_attn(cache, q, p["k"], p["k_scales"], p["v"], p["v_scales"], *batch, out, out_lse=lse)
        elif kind == "window":
            ck.ctkvr_cache_window_attn(cache, q, p["k"], p["v"], *batch, 2000, out, n_sink=5, out_lse=lse, k_scales=p["k_scales"], v_scales=p["v_scales"])
        else:
            ck.ctkvr_cache_tree_attn(cache, q, p["k"], p["v"], *batch, mask, out, out_lse=lse, k_scales=p["k_scales"], v_scales=p["v_scales"])

    first = outputs(st)
    call(*first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = outputs(st)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        call(*again)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    outs, graphs = [outputs(st) for _ in range(2)], []
    torch.cuda.synchronize()
    for o in outs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(*o)
    for i in range(6):
        o = outs[i % 2]
        o[0].zero_(), o[1].zero_()
        graphs[i % 2].replay()
        call(*again)
        assert all(torch.equal(a, b) for a, b in zip(first, o)) and all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("store", STORES)
def test_captured_steps_replay_as_the_sequences_grow(store):
    """A decode step (append, attention, a window, reading the new tokens back) captured once and replayed with lengths that have changed, against the same
    steps run eagerly."""
    st = Q.QuantSetup(32, store, "bf16", 8, 2, 16, (200, 331), (1, 1), spare_cols=2)
    for b, c in ((0, 13), (1, 21)):
        st.table[b, c:c + 2] = torch.tensor([st.num_pages, st.num_pages + 1], dtype=torch.int32)
        st.num_pages += 2
    for name in ("k", "v", "k_scales", "v_scales"):
        x = getattr(st, name)
        setattr(st, name, torch.cat([x.view(torch.uint8), torch.zeros((4,) + x.view(torch.uint8).shape[1:], dtype=torch.uint8)]).view(x.dtype))
    steps = 12
    qs, ks, vs = (torch.randn((steps, 2, n, 128), generator=st.gen).bfloat16().to(DEV) for n in (8, 2, 2))
    out_table = torch.tensor([[0], [1]], dtype=torch.int32, device=DEV)

    def state():
        s = {n: t.clone() for n, t in pages_of(st).items()}
        s.update(q=torch.zeros_like(qs[0]), kn=torch.zeros_like(ks[0]), vn=torch.zeros_like(vs[0]), cur=dev(st.cur).clone(), before=dev(st.cur).clone(),
                 cu=dev(st.cu), table=dev(st.table), cache=cache_of(st), out=torch.zeros_like(qs[0]), lse=torch.zeros((2, 8), device=DEV),
                 near=torch.zeros_like(qs[0]), plain=torch.zeros((2, 2, 2, 16, 128), dtype=torch.bfloat16, device=DEV))
        return s

    def step(s):
        codes, batch = (s["k"], s["k_scales"], s["v"], s["v_scales"]), (s["cu"], s["cur"], s["table"])
        ck.ctkvr_cache_quant_append(s["cache"], s["q"], s["kn"], s["vn"], *batch, s["q"], *codes)
        ck.ctkvr_cache_quant_attn(s["cache"], s["q"], *codes, *batch, s["out"], out_lse=s["lse"])
        ck.ctkvr_cache_window_attn(s["cache"], s["q"], s["k"], s["v"], *batch, 64, s["near"], n_sink=4, k_scales=s["k_scales"], v_scales=s["v_scales"])
        ck.ctkvr_cache_quant_read(s["cache"], *codes, s["cur"], s["table"], out_table, *s["plain"], first_tokens=s["before"])

    def load(s, i):
        s["q"].copy_(qs[i]), s["kn"].copy_(ks[i]), s["vn"].copy_(vs[i])
        s["cur"].copy_(st.cur + i), s["before"].copy_(st.cur + i - 1)

    eager, graphed, warm = state(), state(), state()
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
        for name in ("out", "lse", "near", "plain", "k", "v", "k_scales", "v_scales"):
            assert torch.equal(eager[name].view(torch.uint8), graphed[name].view(torch.uint8)), (i, name)
    assert torch.isfinite(eager["out"]).all() and eager["plain"][:, :, :, 0].abs().sum() > 0


# ---- together -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompts_in_chunks_a_draft_its_accepted_tokens_and_an_index_on_what_is_read_back(store, dtype):
    """Two prompts enter in chunks, a tree of drafted tokens is attended with and one of its paths kept (appended again behind the prompt), a decode step attends over
    all and in a window, and the rows are read back for an index that serves a step with every centroid probed."""
    h, g, page, lens = 8, 2, 16, [300, 220]
    r = torch.Generator().manual_seed(77)
    st = Q.QuantSetup(41, store, dtype, h, g, page, (340, 260), (0, 0))
    cache, table = cache_of(st, max_new=400), dev(st.table)
    p = {n: torch.zeros_like(t) if t.dtype == torch.float32 else torch.zeros_like(t.view(torch.uint8)).view(t.dtype) for n, t in pages_of(st).items()}
    codes = [p[n] for n in ("k", "k_scales", "v", "v_scales")]

    def load():
        for n, t in p.items():
            setattr(st, n, t.cpu())

    def tokens(new, cur, positions=None, rows=None):
        """Appended: the rotated queries, with the Setup at this step."""
        total = sum(new)
        st.new, st.lens, st.total = list(new), list(cur), total
        st.cu, st.cur = torch.tensor([0, new[0], total], dtype=torch.int32), torch.tensor(cur, dtype=torch.int32)
        q, kn, vn = rows or (torch.randn((total, n, 128), generator=r).to(st.td).to(DEV) for n in (h, g, g))
        q_out = torch.empty_like(q)
        ck.ctkvr_cache_quant_append(cache, q, kn, vn, dev(st.cu), dev(st.cur), table, q_out, *codes, positions=dev(positions))
        st.q = q_out.cpu()
        load()
        return q_out, (q, kn, vn)

    def attend(q):
        got = outputs(st)
        ck.ctkvr_cache_quant_attn(cache, q, *codes, dev(st.cu), dev(st.cur), table, got[0], out_lse=got[1])
        return check(st, got, lambda b: Q.sees_range(st, b))

    done, tail = [0, 0], [[], []]
    for new in ((100, 130), (150, 1), (50, 89)):
        done = [d + n for d, n in zip(done, new)]
        q, _ = tokens(new, done)
        attend(q)
        for b in range(2):
            tail[b].append(q[int(st.cu[b]):int(st.cu[b + 1])])
    assert done == lens
    # a draft of 20 and 7 tokens
    new = (20, 7)
    trees = [Q.tree(n, r, 3, 1) for n in new]
    mask, depth = torch.cat([t[0] for t in trees]), [d for _, d in trees]
    positions = torch.tensor([[s + d for s, ds in zip(lens, depth) for d in ds]], dtype=torch.int32)
    q, rows = tokens(new, [s + n for s, n in zip(lens, new)], positions)
    got = outputs(st)
    ck.ctkvr_cache_tree_attn(cache, q, p["k"], p["v"], dev(st.cu), dev(st.cur), table, dev(mask), got[0], out_lse=got[1], k_scales=p["k_scales"],
                             v_scales=p["v_scales"])
    drafted = check(st, got, lambda b: Q.sees_tree(st, b, mask))
    # the deepest token's path is kept: its tokens once more, in order
    kept = []
    for b, (n, ds) in enumerate(zip(new, depth)):
        deep = ds.index(max(ds))
        kept.append([int(st.cu[b]) + j for j in range(n) if int(trees[b][0][deep, 0]) >> j & 1])
    pick = torch.tensor(kept[0] + kept[1], device=DEV)
    q, _ = tokens([len(x) for x in kept], [s + len(x) for s, x in zip(lens, kept)], None, [x[pick] for x in rows])
    # a kept token has seen the same keys at the same positions as in the draft: the definitions agree on the rows that the appends have left
    assert (attend(q) - drafted[pick.cpu()]).abs().max() <= 1e-9
    lens = list(st.lens)
    # one more token: over all keys, and in a window
    lens = [s + 1 for s in lens]
    q, _ = tokens((1, 1), lens)
    attend(q)
    got = outputs(st)
    ck.ctkvr_cache_window_attn(cache, q, p["k"], p["v"], dev(st.cu), dev(st.cur), table, 50, got[0], n_sink=4, out_lse=got[1], k_scales=p["k_scales"],
                               v_scales=p["v_scales"])
    check(st, got, lambda b: Q.sees_window(st, b, 50, 4))
    # rows read back, an index on them, and a decode step with every centroid probed and every key kept
    k, v = (torch.zeros((st.num_pages, g, page, 128), dtype=st.td, device=DEV) for _ in range(2))
    ck.ctkvr_cache_quant_read(cache, *codes, dev(st.cur), table, table, k, v)
    C, budget = 8, min(lens)
    b = lens.index(budget)
    q_tail = torch.cat([torch.cat(tail[b])[-C:] for b in range(2)]).contiguous()
    params = ck.Params(batch=2, n_q_heads=h, n_kv_heads=g, page_size=page, dtype=ck.BF16 if dtype == "bf16" else ck.F32, n_centroids=C, list_len=budget,
                       n_probe=C, top_k=budget)
    idx = ck.ctkvr_build_index(params, q_tail, [0, C, 2 * C], True, k, table, lens)
    sparse, ncand = torch.empty((2, h, 128), device=DEV), torch.empty((2, g), dtype=torch.int32, device=DEV)
    ck.ctkvr_decode_step(idx, q, k, v, table, sparse, out_ncand=ncand)
    assert (ncand[b] == budget).all()
    want, _, tol, _ = Q.attention(st, lambda b: Q.sees_range(st, b))
    for kv in range(g):
        # keys and values that are read back are rounded to the type: a score moves by as much of the sum of its products' sizes, the probabilities with it
        keys, values = (st.held(name, b, kv, lens[b])[0] for name in ("k", "v"))
        heads = slice(kv * h // g, (kv + 1) * h // g)
        moved = float((st.q[b, heads].to(O.F8).abs() @ keys.abs().T).max()) / math.sqrt(128.0) * O.HALF[dtype]
        allowed = tol[b, heads] + (math.expm1(2 * moved) + O.HALF[dtype]) * values.abs().max()
        assert ((sparse[b, heads].cpu().to(O.F8) - want[b, heads]).abs() <= allowed).all()
    ck.ctkvr_free(idx)
