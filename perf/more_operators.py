"""Measured cases of what a paged KV cache of 8-bit rows and of drafted tokens needs: rows quantised as they are appended and read back, attention over
quantised rows, attention in a sliding window beside the first tokens, attention of a tree of drafted tokens.

Where ``own`` is false ``run`` computes an operator in its plain form, elementary torch operations in 32 bits (angles in 64) on the gathered
rows; where it is true it calls the library.  Contexts, head shapes and page sizes are those of the repository's workloads (32K tokens, 32 query
heads on 8 KV heads, pages of 16) and ranges around them.  Keys are N(0, 1) with RoPE, values N(0, 1), queries N(0, 1) scaled by 2 so that
attention is neither flat nor on a single key; the pages lie in a random order.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"
D = 128
BASE = 10000.0
TOP = {"int8": 127.0, "fp8": 448.0}     # the largest code
CODES = {"int8": torch.int8, "fp8": torch.float8_e4m3fn}

_DEFAULTS = {
    "op": "attn",        # append | read | attn | window | tree
    "store": "int8",     # what the cache holds: plain (rows of dtype; window and tree only), int8 or fp8 codes with a scale a row
    "dtype": "bf16", "h": 32, "g": 8, "page": 16, "batch": 1, "len_seed": 0,
    "ctx_lo": 32768, "ctx_hi": 32768,     # tokens in the cache, the new ones among them: uniform in [ctx_lo, ctx_hi]
    "new_lo": 1, "new_hi": 1,             # new tokens of a sequence (read: the tokens that are read, the last ones)
    "cap": 0.0,          # attn, window, tree: scores capped to cap * tanh(z / cap)
    "bias": False,       # attn, window: ... minus a slope per head times the distance
    "docs": 0,           # attn: tokens of a document see only it: documents of about so many tokens (0: no document mask)
    "prefix": 0,         # attn: tokens at the start that every token sees
    "window": 0, "sinks": 0,    # window: the last tokens that a token sees, itself among them, and the first ones
    "branch": 4,         # tree: a drafted token follows one of the so many drafted before it
}


def _case(name, **over):
    return dict(_DEFAULTS, name=name, **over)


def listed():
    return [
        # one decoded token of 16 running requests goes into the cache and comes back as the plain row that the newest tokens are kept in beside it
        _case("append_1x16_int8", op="append", batch=16, ctx_lo=2048, ctx_hi=4096, len_seed=1),
        # a prompt's chunk of 8K tokens, written as 8-bit floats, and the pages that its index is built on
        _case("append_8k_fp8", op="append", store="fp8", ctx_lo=16384, ctx_hi=16384, new_lo=8192, new_hi=8192),
        # a 32K context read back into plain pages, to build an index on or to hand it on
        _case("read_32k_int8", op="read", new_lo=32768, new_hi=32768),
        # the unequal ends of a small batch of fp32 rows
        _case("read_ragged_f32_fp8", op="read", store="fp8", dtype="f32", h=8, g=2, batch=3, ctx_lo=900, ctx_hi=5000, new_lo=300, new_hi=900, len_seed=5),
        # a short prompt in fp32 on a small model, every token of the first 100 visible to all
        _case("attn_500_f32_int8", dtype="f32", h=8, g=2, ctx_lo=500, ctx_hi=500, new_lo=500, new_hi=500, prefix=100),
        # the dense decode step of one request at 32K
        _case("attn_1_of_32k_int8"),
        # ... of a running batch of unequal lengths, with capped scores
        _case("attn_1x16_ragged_fp8", store="fp8", batch=16, ctx_lo=8192, ctx_hi=65536, len_seed=4, cap=30.0),
        # the last chunk of a 32K prompt: the largest case
        _case("attn_2k_of_32k_fp8", store="fp8", new_lo=2048, new_hi=2048),
        # a decode step of a layer that sees the last 4096 tokens and the first 4, of a running batch of unequal lengths
        _case("window_1x16", op="window", store="plain", batch=16, ctx_lo=8192, ctx_hi=65536, len_seed=4, window=4096, sinks=4),
        # a whole prompt of 8K tokens in such a layer, of a window of 1024
        _case("window_8k", op="window", store="plain", ctx_lo=8192, ctx_hi=8192, new_lo=8192, new_hi=8192, window=1024, sinks=4),
        # one request's draft of 64 tokens at 32K
        _case("tree_64_of_32k", op="tree", store="plain", new_lo=64, new_hi=64),
        # drafts of 8 to 25 tokens of a running batch on 8-bit rows
        _case("tree_8x_ragged_int8", op="tree", batch=8, ctx_lo=3000, ctx_hi=20000, new_lo=8, new_hi=25, len_seed=7, branch=3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    c = dict(_DEFAULTS)
    op = c["op"] = rng.choice(["append", "read", "attn", "attn", "attn", "window", "window", "tree", "tree"])
    c["store"] = rng.choice(["int8", "fp8"] if op in ("append", "read", "attn") else ["plain", "plain", "int8", "fp8"])
    # (an appended row's codes are compared as bf16 values: a code next to a border may go to either side of it)
    f32 = op != "append" and rng.random() < 0.2
    c["dtype"] = "f32" if f32 else "bf16"
    c["h"], c["g"] = rng.choice([(32, 8), (32, 8), (32, 4), (8, 2), (8, 8), (16, 8), (40, 10)])
    c["page"] = rng.choice([16, 16, 32, 64])
    c["batch"] = rng.choice([1, 1, 2, 3, _log_int(rng, 4, 16)])
    c["len_seed"] = rng.randrange(1 << 20)
    hi = min(32768 if f32 else 131072, (131072 if f32 else 524288) // c["batch"])
    most = 1 << 22 if f32 else 1 << 26          # pairs of new tokens and keys of the largest listed case
    if op == "append":
        c["ctx_hi"] = _log_int(rng, 64, min(hi, 65536 // c["batch"]))
        c["new_hi"] = 1 if rng.random() < 0.3 else _log_int(rng, 1, min(c["ctx_hi"], 8192 // c["batch"]))
    elif op == "read":
        c["ctx_hi"] = _log_int(rng, 64, min(hi, 65536 // c["batch"]))
        c["new_hi"] = _log_int(rng, 1, c["ctx_hi"])
    elif op == "tree":
        c["ctx_hi"] = _log_int(rng, 128, hi)
        c["new_hi"] = min(max(1, most // (c["batch"] * c["ctx_hi"])), _log_int(rng, 2, 128))
        c["branch"] = rng.choice([1, 2, 4, 8])
    else:
        c["ctx_hi"] = _log_int(rng, 64, hi)
        c["new_hi"] = 1 if rng.random() < 0.35 else _log_int(rng, 1, max(1, min(c["ctx_hi"], most // (c["batch"] * c["ctx_hi"]))))
        c["bias"] = rng.random() < 0.2
    c["new_lo"] = 1 if rng.random() < 0.5 else c["new_hi"]
    c["ctx_lo"] = max(c["new_hi"], c["ctx_hi"] // rng.choice([1, 1, 2, 5]))
    if op in ("attn", "window", "tree"):
        c["cap"] = rng.choice([0.0, 0.0, 30.0, 50.0])
    if op == "attn":
        c["docs"] = rng.choice([0, 0, 0, _log_int(rng, 50, 5000)])
        c["prefix"] = rng.choice([0, 0, 0, _log_int(rng, 1, c["ctx_hi"])])
    if op == "window":
        c["window"] = _log_int(rng, 1, min(8192, c["ctx_hi"]))
        c["sinks"] = rng.choice([0, 1, 4, 4, _log_int(rng, 5, 200)])
    return c


# ------------------------------------------------------------------------------
# sizes
# ------------------------------------------------------------------------------
def _lens(case):
    """(tokens in the cache, new tokens) of every sequence."""
    r = np.random.RandomState(case["len_seed"])
    ctx = [int(x) for x in r.randint(case["ctx_lo"], case["ctx_hi"] + 1, size=case["batch"])]
    new = [min(s, int(x)) for s, x in zip(ctx, r.randint(case["new_lo"], case["new_hi"] + 1, size=case["batch"]))]
    return ctx, new


def _first_key(case, s, n):
    """First key that each of a sequence's n last tokens sees: where its document begins."""
    pos = np.arange(s - n, s)
    if not case["docs"]:
        return np.zeros(n, np.int64)
    r = np.random.RandomState(case["len_seed"] + s)
    starts = np.concatenate([[0], np.cumsum(r.randint(case["docs"] // 2 + 1, 2 * case["docs"] + 1, size=2 * s // max(1, case["docs"]) + 2))])
    return starts[np.searchsorted(starts, pos, side="right") - 1]


def _tree(case, b, n):
    """The drafted tokens that each of a sequence's n drafted ones sees, itself among them, as rows of truth values."""
    r = np.random.RandomState(case["len_seed"] + 7919 * b + 1)
    sees = np.zeros((n, n), bool)
    for i in range(n):
        if i:
            sees[i] = sees[r.randint(max(0, i - case["branch"]), i)]
        sees[i, i] = True
    return sees


def _pairs(case):
    """Visible (token, key) pairs, and keys that some token sees."""
    pairs = keys = 0
    ctx, new = _lens(case)
    for b, (s, n) in enumerate(zip(ctx, new)):
        pos = np.arange(s - n, s)
        if case["op"] == "tree":
            pairs += n * (s - n) + int(_tree(case, b, n).sum())
            keys += s
        elif case["op"] == "window":
            first = np.maximum(pos + 1 - case["window"], 0)
            pairs += int((pos + 1 - first + np.minimum(first, case["sinks"])).sum())
            keys += int(s - first[0] + min(first[0], case["sinks"]))
        else:
            first, end = _first_key(case, s, n), np.maximum(pos + 1, min(case["prefix"], s))
            pairs += int(np.maximum(end - first, 0).sum())
            keys += int(end.max() - first.min())
    return pairs, keys


def work(case):
    case = dict(_DEFAULTS, **case)
    e = 2 if case["dtype"] == "bf16" else 4
    row = D * e if case["store"] == "plain" else D + 4
    h, g = case["h"], case["g"]
    n = sum(_lens(case)[1])
    if case["op"] == "append":   # queries, keys and values in and out; the rows' codes and scales out and in; their values out
        return {"bytes": n * ((2 * h + 4 * g) * D * e + 4 * g * row), "flops": n * (h + g) * D * 3.0}
    if case["op"] == "read":     # codes and scales in, values out
        return {"bytes": n * 2 * g * (row + D * e), "flops": n * 2.0 * g * D}
    pairs, keys = _pairs(case)   # queries, visible keys and values (and the drafts' masks) in; outputs and log-sum-exps out
    return {"bytes": keys * g * 2 * row + n * h * (2 * D * e + 4) + (sum(4 * m * -(-m // 32) for m in _lens(case)[1]) if case["op"] == "tree" else 0),
            "flops": 4.0 * D * h * pairs}


# ------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------
def _rope(x, pos):
    theta = BASE ** (-torch.arange(64, dtype=torch.float64, device=x.device) / 64.0)
    ang = pos.to(torch.float64)[:, None] * theta          # (32 bits lose the angles of far positions)
    c, s = torch.cos(ang).float()[:, None, :], torch.sin(ang).float()[:, None, :]
    a, b = x[..., :64], x[..., 64:]
    return torch.cat([a * c - b * s, b * c + a * s], dim=-1)


def _quantised(x, store):
    """Codes of rows of 128 and a scale for each: the largest magnitude becomes the largest code."""
    amax = x.abs().amax(dim=-1, keepdim=True)
    y = torch.where(amax > 0, x * TOP[store] / amax, 0.0)
    return (y.round() if store == "int8" else y).to(CODES[store]), (amax / TOP[store]).squeeze(-1)


def _dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV, dtype)


def _mask_words(case, new):
    """Bit j of a drafted token's row: it sees the j-th drafted token of its sequence."""
    words = max(1, -(-max(new) // 32))
    rows = []
    for b, n in enumerate(new):
        sees = np.zeros((n, words, 32), np.uint64)
        sees.reshape(n, -1)[:, :n] = _tree(case, b, n)
        rows.append((sees << np.arange(32, dtype=np.uint64)).sum(axis=-1))
    return np.concatenate(rows).astype(np.uint32).view(np.int32)


def prepare(case, seed):
    case = dict(_DEFAULTS, **case)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    h, g, page, batch, op = case["h"], case["g"], case["page"], case["batch"], case["op"]
    ctx, new = _lens(case)
    n = sum(new)
    pages = [-(-s // page) for s in ctx]
    pool, cols = sum(pages) + 3, max(pages)
    perm = torch.randperm(pool, generator=gen, device=DEV)
    k = torch.randn((pool, g, page, D), generator=gen, device=DEV).to(dt)
    v = torch.randn((pool, g, page, D), generator=gen, device=DEV).to(dt)
    table = torch.full((batch, cols), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, (s, m, p) in enumerate(zip(ctx, new, pages)):
        phys = perm[at:at + p]
        at += p
        table[b, :p] = phys.to(torch.int32)
        if op != "append":
            pos = torch.arange(p * page, device=DEV)
            if op == "tree":     # a drafted token stands behind those that it sees
                pos[s - m:s] = s - m - 1 + _dev(_tree(case, b, m).sum(axis=1), torch.long)
            rows = _rope(k[phys].float().transpose(1, 2).reshape(p * page, g, D), pos)
            k[phys] = rows.view(p, page, g, D).transpose(1, 2).to(dt)
    st = {"case": case, "table": table, "cu": _dev(np.concatenate([[0], np.cumsum(new)])), "cur": _dev(ctx), "ctx": ctx, "new": new,
          "k": k, "v": v, "k_scales": None, "v_scales": None}
    if case["store"] != "plain":
        (st["k"], st["k_scales"]), (st["v"], st["v_scales"]) = _quantised(k.float(), case["store"]), _quantised(v.float(), case["store"])
    if op == "append":           # views of one fused projection
        qkv = torch.randn((n, (h + 2 * g) * D), generator=gen, device=DEV).to(dt)
        st["q"], st["kn"], st["vn"] = (t.view(n, -1, D) for t in torch.split(qkv, [h * D, g * D, g * D], dim=1))
        st["q_out"] = torch.zeros((n, h, D), dtype=dt, device=DEV)
    if op in ("append", "read"):   # plain pages for the tokens that are read, from the first slot on
        out_pages = [-(-m // page) for m in new]
        st["out_table"] = torch.full((batch, max(out_pages)), -1, dtype=torch.int32, device=DEV)
        perm, at = torch.randperm(sum(out_pages) + 1, generator=gen, device=DEV).to(torch.int32), 0
        for b, p in enumerate(out_pages):
            st["out_table"][b, :p] = perm[at:at + p]
            at += p
        st["k_out"] = torch.zeros((sum(out_pages) + 1, g, page, D), dtype=dt, device=DEV)
        st["v_out"] = torch.zeros_like(st["k_out"])
        st["first"] = _dev(np.subtract(ctx, new))
    else:
        depth = [np.arange(m) if op != "tree" else _tree(case, b, m).sum(axis=1) - 1 for b, m in enumerate(new)]
        pos = _dev(np.concatenate([s - m + d for s, m, d in zip(ctx, new, depth)]), torch.long)
        st["q"] = _rope(2.0 * torch.randn((n, h, D), generator=gen, device=DEV), pos).to(dt)
        st["slopes"] = _dev(2.0 ** (-8.0 * np.arange(1, h + 1) / h), torch.float32) if case["bias"] else None
        st["first"] = _dev(np.concatenate([_first_key(case, s, m) for s, m in zip(ctx, new)])) if case["docs"] else None
        st["prefix"] = _dev(np.minimum(case["prefix"], ctx)) if case["prefix"] else None
        st["mask"] = _dev(_mask_words(case, new)) if op == "tree" else None
        st["out"] = torch.zeros((n, h, D), dtype=dt, device=DEV)
        st["lse"] = torch.zeros((n, h), dtype=torch.float32, device=DEV)
    if own:
        import paper_2512_15550_amd as ck
        st["cache"] = ck.ctkvr_cache_create(ck.CacheParams(
            batch=batch, n_q_heads=h, n_kv_heads=g, page_size=page, dtype=ck.BF16 if case["dtype"] == "bf16" else ck.F32, num_pages=pool,
            max_pages=cols, max_new=max(n, 1), softcap=case["cap"], rope_base=BASE))
    return st


# ------------------------------------------------------------------------------
# the plain forms
# ------------------------------------------------------------------------------
def _token(st, n):
    """Sequence and slot of every new token."""
    cu, cur = st["cu"].long(), st["cur"].long()
    t = torch.arange(n, device=DEV)
    b = torch.searchsorted(cu, t, right=True) - 1
    return b, cur[b] - cu[b + 1] + t


def _rows(pages, scales, table, key, page):
    """Rows `key` [batch][keys] of every sequence, [batch][g][keys][128] in 32 bits."""
    b, kv = torch.arange(key.shape[0], device=DEV)[:, None, None], torch.arange(pages.shape[1], device=DEV)[None, :, None]
    key = key[:, None, :]
    phys = table.long()[b, key // page].clamp(min=0)
    x = pages[phys, kv, key % page].float()
    return x if scales is None else x * scales[phys, kv, key % page][..., None]


def _keys(st):
    """The keys that some new token of a sequence may see, [batch][keys], ascending and each once; -1: none."""
    case, slots = st["case"], st["table"].shape[1] * st["case"]["page"]
    reach = case["window"] + max(st["new"]) - 1
    if case["op"] != "window" or reach + case["sinks"] >= slots:
        return torch.arange(slots, device=DEV).expand(case["batch"], -1)
    start = (st["cur"].long() - reach)[:, None]
    near = start + torch.arange(reach, device=DEV)
    early = torch.arange(case["sinks"], device=DEV).expand(case["batch"], -1)
    return torch.cat([torch.where(early < start, early, -1), torch.where(near >= 0, near, -1)], dim=1)


def _attn(st):
    """Attention of a batch padded to its longest chunk: scores [batch][g][new][G][keys]."""
    case = st["case"]
    g, group, n_max, page = case["g"], case["h"] // case["g"], max(st["new"]), case["page"]
    b, slot = _token(st, st["q"].shape[0])
    i = torch.arange(b.numel(), device=DEV) - st["cu"].long()[b]
    key = _keys(st)
    k = _rows(st["k"], st["k_scales"], st["table"], key.clamp(min=0), page)
    q = torch.zeros((case["batch"], n_max, g, group, D), device=DEV)
    q[b, i] = st["q"].float().view(-1, g, group, D)
    z = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(case["batch"], g, n_max * group, D), k.transpose(2, 3).contiguous())
    z = z.view(case["batch"], g, n_max, group, -1).mul_(1.0 / math.sqrt(D))
    if case["cap"]:
        z = z.div_(case["cap"]).tanh_().mul_(case["cap"])
    pos = torch.full((case["batch"], n_max), -1, dtype=torch.long, device=DEV)
    pos[b, i] = slot
    key = key[:, None, :]
    if st["slopes"] is not None:
        far = (pos[:, :, None] - key).abs().float()
        z -= st["slopes"].view(1, g, 1, group, 1) * far[:, None, :, None, :]
    if case["op"] == "tree":     # what stands before the draft, and the draft's tokens by their bits
        word = torch.zeros((case["batch"], n_max, st["mask"].shape[1]), dtype=torch.int32, device=DEV)
        word[b, i] = st["mask"]
        drafted = (word[..., None] >> torch.arange(32, device=DEV, dtype=torch.int32) & 1).flatten(2).bool()
        j = key - (st["cur"] - st["cu"][1:] + st["cu"][:-1]).long()[:, None, None]
        seen = torch.gather(drafted, 2, j.clamp(0, drafted.shape[2] - 1).expand(-1, n_max, -1)) & (j < drafted.shape[2]) | (j < 0)
    else:
        seen = key <= pos[:, :, None]
    if st["prefix"] is not None:
        seen |= key < st["prefix"][:, None, None]
    if st["first"] is not None:
        first = torch.zeros_like(pos)
        first[b, i] = st["first"].long()
        seen &= key >= first[:, :, None]
    if case["op"] == "window":
        seen &= (key > pos[:, :, None] - case["window"]) | (key < case["sinks"])
    seen &= (key < st["cur"][:, None, None]) & (key >= 0)
    seen &= (pos >= 0)[:, :, None]
    z.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    m = z.amax(dim=-1, keepdim=True).clamp_(min=-1e30)
    p = z.sub_(m).exp_()
    l = p.sum(dim=-1, keepdim=True)
    v = _rows(st["v"], st["v_scales"], st["table"], key[:, 0].clamp(min=0), page)
    o = torch.matmul(p.view(case["batch"], g, n_max * group, -1), v).view(case["batch"], g, n_max, group, D) / l.clamp(min=1e-30)
    st["out"].copy_(o[b, :, i].reshape(st["out"].shape))
    st["lse"].copy_((torch.log(l) + m)[b, :, i].reshape(st["lse"].shape))
    return st["out"], st["lse"]


def _append(st):
    case = st["case"]
    b, slot = _token(st, st["q"].shape[0])
    st["q_out"].copy_(_rope(st["q"].float(), slot))
    page, at = st["table"][b, slot // case["page"]].long(), slot % case["page"]
    for name, x in (("k", _rope(st["kn"].float(), slot)), ("v", st["vn"].float())):
        codes, scales = _quantised(x, case["store"])
        st[name].view(torch.uint8)[page, :, at] = codes.view(torch.uint8)
        st[name + "_scales"][page, :, at] = scales


def _read(st):
    page = st["case"]["page"]
    b, slot = _token(st, sum(st["new"]))
    j = slot - st["first"].long()[b]
    src, dst = st["table"][b, slot // page].long(), st["out_table"][b, j // page].long()
    for name in ("k", "v"):
        x = st[name].view(torch.uint8)[src, :, slot % page].view(st[name].dtype)
        st[name + "_out"][dst, :, j % page] = (x.float() * st[name + "_scales"][src, :, slot % page][..., None]).to(st[name + "_out"].dtype)


def run(st):
    op = st["case"]["op"]
    if own:
        import paper_2512_15550_amd as ck
        case, cache = st["case"], st["cache"]
        batch = st["cu"], st["cur"], st["table"]
        codes = st["k"], st["k_scales"], st["v"], st["v_scales"]
        if op == "append":
            ck.ctkvr_cache_quant_append(cache, st["q"], st["kn"], st["vn"], *batch, st["q_out"], *codes)
        if op in ("append", "read"):
            ck.ctkvr_cache_quant_read(cache, *codes, st["cur"], st["table"], st["out_table"], st["k_out"], st["v_out"], first_tokens=st["first"])
        elif op == "attn":
            ck.ctkvr_cache_quant_attn(cache, st["q"], *codes, *batch, st["out"], out_lse=st["lse"], slopes=st["slopes"], prefix_lens=st["prefix"],
                                      first_key=st["first"])
        elif op == "window":
            ck.ctkvr_cache_window_attn(cache, st["q"], st["k"], st["v"], *batch, case["window"], st["out"], n_sink=case["sinks"], out_lse=st["lse"],
                                       slopes=st["slopes"], k_scales=st["k_scales"], v_scales=st["v_scales"])
        else:
            ck.ctkvr_cache_tree_attn(cache, st["q"], st["k"], st["v"], *batch, st["mask"], st["out"], out_lse=st["lse"], k_scales=st["k_scales"],
                                     v_scales=st["v_scales"])
    elif op in ("append", "read"):
        if op == "append":
            _append(st)
        _read(st)
    else:
        _attn(st)
    if op == "append":
        return st["q_out"], st["k_out"], st["v_out"]
    return (st["k_out"], st["v_out"]) if op == "read" else (st["out"], st["lse"])


# ------------------------------------------------------------------------------
# from the definitions in 64 bits, sequence by sequence
# ------------------------------------------------------------------------------
def _values(x, store):
    """The values that rows x [..., 128] in 64 bits stand for once they are quantised: the nearest code, ties to even, times the scale."""
    amax = x.abs().amax(dim=-1, keepdim=True)
    y, scale = torch.where(amax > 0, x * TOP[store] / amax, 0.0), amax / TOP[store]
    if store == "int8":
        return torch.round(y) * scale
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3.0)     # 3 bits behind the leading one, exponents from -6 on
    return torch.round(y / step) * step * scale


def exact(case, seed):
    global own
    case, before = dict(_DEFAULTS, **case), own
    own = False
    try:
        st = prepare(case, seed)
    finally:
        own = before
    f8 = torch.float64
    ctx, new, g, h, page, op = st["ctx"], st["new"], case["g"], case["h"], case["page"], case["op"]
    cu = [0] + [int(x) for x in np.cumsum(new)]

    def held(name, b, t):
        """Rows t of sequence b, [keys][g][128], as the cache holds them."""
        phys = st["table"][b, t // page].long()
        x = st[name][phys].to(torch.float32).to(f8)[torch.arange(t.numel(), device=DEV), :, t % page]
        scales = st[name + "_scales"]
        return x if scales is None else x * scales[phys, :, t % page].to(f8)[..., None]

    if op in ("append", "read"):
        outs = [st["k_out"].to(f8), st["v_out"].to(f8)]
        if op == "append":
            pos = np.concatenate([np.arange(s - n, s) for s, n in zip(ctx, new)])
            turn = torch.from_numpy(np.exp(1j * pos[:, None] * BASE ** (-np.arange(64) / 64.0))).to(DEV)[:, None, :]

            def rotated(x):
                y = torch.complex(x[..., :64].to(f8), x[..., 64:].to(f8)) * turn
                return torch.cat([y.real, y.imag], dim=-1)

            rows = [_values(rotated(st["kn"]), case["store"]), _values(st["vn"].to(f8), case["store"])]
        for b, (s, n) in enumerate(zip(ctx, new)):
            j = torch.arange(n, device=DEV)
            for i, name in enumerate(("k", "v")):
                x = rows[i][cu[b]:cu[b + 1]] if op == "append" else held(name, b, s - n + j)
                outs[i][st["out_table"][b, j // page].long(), :, j % page] = x
        return (rotated(st["q"]), *outs) if op == "append" else tuple(outs)

    step = max(1, (1 << 28) // (h * max(ctx)))
    out, lse = torch.zeros((sum(new), h, D), dtype=f8, device=DEV), torch.zeros((sum(new), h), dtype=f8, device=DEV)
    for b, (s, n) in enumerate(zip(ctx, new)):
        sees = torch.from_numpy(_tree(case, b, n)).to(DEV) if op == "tree" else None
        docs = _dev(_first_key(case, s, n), torch.long)
        k_all = v_all = None
        for i in range(0, n, step):
            m = min(step, n - i)
            pos = torch.arange(s - n + i, s - n + i + m, device=DEV)
            key = torch.arange(s, device=DEV)
            if op == "window":
                lo = max(0, s - n + i + 1 - case["window"])
                key = torch.cat([torch.arange(min(lo, case["sinks"]), device=DEV), torch.arange(lo, s - n + i + m, device=DEV)])
            if op == "window" or k_all is None:
                k_all, v_all = held("k", b, key).transpose(0, 1).contiguous(), held("v", b, key).transpose(0, 1).contiguous()
            q = st["q"][cu[b] + i:cu[b] + i + m].to(f8).view(m, g, h // g, D).permute(1, 2, 0, 3).reshape(g, -1, D)
            z = torch.bmm(q, k_all.transpose(1, 2).contiguous()).view(g, h // g, m, -1) / math.sqrt(D)
            if case["cap"]:
                z = case["cap"] * torch.tanh(z / case["cap"])
            if case["bias"]:
                z = z - st["slopes"].to(f8).view(g, h // g, 1, 1) * (pos[:, None] - key).abs().to(f8)
            if op == "tree":
                hidden = torch.zeros((m, s), dtype=torch.bool, device=DEV)
                hidden[:, s - n:] = ~sees[i:i + m]
            elif op == "window":
                hidden = (key > pos[:, None]) | ((pos[:, None] - key >= case["window"]) & (key >= case["sinks"]))
            else:
                hidden = (key > pos[:, None]) & (key >= min(case["prefix"], s)) | (key < docs[i:i + m, None])
            z = z.masked_fill(hidden, -math.inf)
            rows = slice(cu[b] + i, cu[b] + i + m)
            lse[rows] = torch.logsumexp(z, dim=-1).permute(2, 0, 1).reshape(m, h)
            p = torch.softmax(z, dim=-1).nan_to_num(0.0).view(g, -1, z.shape[-1])
            out[rows] = torch.bmm(p, v_all).view(g, h // g, m, D).permute(2, 0, 1, 3).reshape(m, h, D)
    return out, lse
