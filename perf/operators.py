"""Measured cases of the operators on the paged KV cache: append with rotary positions, attention of new tokens, accumulated attention
weights, eviction.

Where ``own`` is false ``run`` computes an operator in its plain form, elementary torch operations in 32 bits (angles in 64) on the gathered
cache; where it is true it calls the library.  Contexts, head shapes and page sizes are those of the repository's workloads (32K and
128K tokens, 32 query heads on 8 or 4 KV heads, pages of 16) and ranges around them.  Keys are N(0, 1) with RoPE, values N(0, 1), queries N(0, 1)
scaled by 2 so that attention is neither flat nor on a single key; the pages lie in a random order.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"
D = 128
BASE = 10000.0

_DEFAULTS = {
    "op": "attn",        # append | attn | weights | evict
    "dtype": "bf16", "h": 32, "g": 8, "page": 16, "batch": 1, "len_seed": 0,
    "ctx_lo": 32768, "ctx_hi": 32768,     # tokens in the cache, the new ones among them: uniform in [ctx_lo, ctx_hi]
    "new_lo": 1, "new_hi": 1,             # new tokens of a sequence
    "axes": 1,           # append: position axes (3: time, height, width of an image in the text)
    "cap": 0.0,          # attn, weights: scores capped to cap * tanh(z / cap)
    "bias": False,       # ... minus a slope per head times the distance
    "docs": 0,           # ... tokens of a document see only it: documents of about so many tokens (0: no document mask)
    "prefix": 0,         # ... tokens at the start that every token sees
    "decay": 1.0,        # weights: what is left of the weights so far
    "budget": 0, "n_init": 0, "n_local": 0,   # evict
}


def _case(name, **over):
    return dict(_DEFAULTS, name=name, **over)


def listed():
    return [
        # one decoded token of 16 running requests goes into the cache: launches and latency are all of it
        _case("append_1x16", op="append", batch=16, ctx_lo=2048, ctx_hi=4096, len_seed=1),
        # a prompt's chunk of 8K tokens, text around an image, rotated by time, height and width
        _case("append_8k_3axes", op="append", ctx_lo=16384, ctx_hi=16384, new_lo=8192, new_hi=8192, axes=3),
        # the smallest attention: a short prompt in fp32 on a small model, every token of the first 100 visible to all
        _case("attn_500_f32", dtype="f32", h=8, g=2, ctx_lo=500, ctx_hi=500, new_lo=500, new_hi=500, prefix=100),
        # the dense decode step of one request at 32K, which the sparse step stands beside
        _case("attn_1_of_32k"),
        # ... of a running batch of unequal lengths, with capped scores
        _case("attn_1x16_ragged", batch=16, ctx_lo=8192, ctx_hi=65536, len_seed=4, cap=30.0),
        # the last chunk of a 32K prompt
        _case("attn_2k_of_32k", new_lo=2048, new_hi=2048),
        # several packed documents and a distance bias: a batch of two odd chunks
        _case("attn_docs_bias", batch=2, g=4, ctx_lo=7000, ctx_hi=9000, new_lo=3001, new_hi=5999, len_seed=9, bias=True, docs=2000),
        # the weight of every key under a decoded token, added after its attention
        _case("weights_1_of_32k", op="weights", decay=0.98),
        # the weights of a 128K prompt under its last 64 tokens, before it is cut down
        _case("weights_64_of_128k", op="weights", ctx_lo=131072, ctx_hi=131072, new_lo=64, new_hi=64),
        # ... of two whole prompts under all of their tokens
        _case("weights_prompt", op="weights", batch=2, ctx_lo=4000, ctx_hi=8000, new_lo=4000, new_hi=8000, len_seed=3),
        # a 32K prompt cut down to 4K tokens
        _case("evict_32k_to_4k", op="evict", budget=4096, n_init=4, n_local=512),
        # a running batch at its budget: one token of each goes
        _case("evict_1x16", op="evict", batch=16, ctx_lo=4097, ctx_hi=4097, budget=4096, n_init=4, n_local=512),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    c = dict(_DEFAULTS)
    op = c["op"] = rng.choice(["append", "attn", "attn", "attn", "weights", "weights", "evict"])
    c["dtype"] = "f32" if rng.random() < 0.2 else "bf16"
    c["h"], c["g"] = rng.choice([(32, 8), (32, 8), (32, 4), (8, 2), (8, 8), (16, 8), (40, 10)])
    c["page"] = rng.choice([16, 16, 32, 64])
    c["batch"] = rng.choice([1, 1, 2, 3, _log_int(rng, 4, 16)])
    c["len_seed"] = rng.randrange(1 << 20)
    f32 = c["dtype"] == "f32"
    hi = min(32768 if f32 else 131072, (131072 if f32 else 524288) // c["batch"])
    if op == "append":
        c["ctx_hi"] = _log_int(rng, 64, min(hi, 65536 // c["batch"]))
        c["new_hi"] = 1 if rng.random() < 0.3 else _log_int(rng, 1, min(c["ctx_hi"], 8192 // c["batch"]))
        c["axes"] = rng.choice([1, 3])
    elif op == "attn":
        c["ctx_hi"] = _log_int(rng, 64, hi)
        most = max(1, int((1 << 22 if f32 else 1 << 26) // (c["batch"] * c["ctx_hi"])))   # pairs of the largest listed case
        c["new_hi"] = 1 if rng.random() < 0.35 else _log_int(rng, 1, max(1, min(c["ctx_hi"], most)))
    elif op == "weights":
        c["ctx_hi"] = _log_int(rng, 64, hi)
        most = max(1, int((1 << 22 if f32 else 1 << 25) // (c["batch"] * c["ctx_hi"])))
        c["new_hi"] = 1 if rng.random() < 0.35 else _log_int(rng, 1, max(1, min(c["ctx_hi"], most)))
        c["decay"] = rng.choice([1.0, 0.95])
    else:
        c["ctx_hi"] = _log_int(rng, 64, min(hi, 262144 // c["batch"]))
        c["n_init"], c["n_local"] = rng.choice([(0, 0), (4, 16), (1, 31)])
        c["budget"] = max(1, c["n_init"] + c["n_local"], _log_int(rng, 48, max(49, c["ctx_hi"] // 2)))
        if rng.random() < 0.3:
            c["budget"] = max(c["n_init"] + c["n_local"] + 1, c["ctx_hi"] - 1)
    c["new_lo"] = 1 if rng.random() < 0.5 else c["new_hi"]
    c["ctx_lo"] = max(c["new_hi"], c["ctx_hi"] // rng.choice([1, 1, 2, 5]))
    if op in ("attn", "weights"):
        c["cap"] = rng.choice([0.0, 0.0, 30.0, 50.0])
        c["bias"] = rng.random() < 0.2
        c["docs"] = rng.choice([0, 0, 0, _log_int(rng, 50, 5000)])
        c["prefix"] = rng.choice([0, 0, 0, _log_int(rng, 1, c["ctx_hi"])])
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


def _pairs(case):
    """Visible (token, key) pairs, and keys that some token sees."""
    pairs = keys = 0
    ctx, new = _lens(case)
    for s, n in zip(ctx, new):
        pos, first = np.arange(s - n, s), _first_key(case, s, n)
        end = np.maximum(pos + 1, min(case["prefix"], s))
        pairs += int(np.maximum(end - first, 0).sum())
        keys += int(end.max() - first.min())
    return pairs, keys


def work(case):
    case = dict(_DEFAULTS, **case)
    e = 2 if case["dtype"] == "bf16" else 4
    h, g = case["h"], case["g"]
    ctx, new = _lens(case)
    n = sum(new)
    if case["op"] == "append":   # queries, keys and values in and out
        return {"bytes": n * ((2 * h + 4 * g) * D * e + 4 * (case["axes"] if case["axes"] > 1 else 0)), "flops": n * (h + g) * D * 3.0}
    if case["op"] == "evict":    # weights in; kept rows that move in and out; weights and ids out
        nbytes = 0.0
        for s in ctx:
            m, mid = min(s, case["budget"]), s - case["n_init"] - case["n_local"]
            moved = max(0.0, m - case["n_init"] - mid / (s - m + 1.0)) if s > m else 0.0
            nbytes += g * (4 * s + moved * 4 * D * e + 8 * m)
        return {"bytes": nbytes, "flops": 0}
    pairs, keys = _pairs(case)
    if case["op"] == "attn":     # queries, visible keys and values in; outputs and log-sum-exps out
        return {"bytes": keys * g * 2 * D * e + n * h * (2 * D * e + 4), "flops": 4.0 * D * h * pairs}
    return {"bytes": keys * g * D * e + sum(ctx) * g * 8 + n * h * (D * e + 4), "flops": 2.0 * D * h * pairs}


# ------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------
def _rope(x, pos):
    theta = BASE ** (-torch.arange(64, dtype=torch.float64, device=x.device) / 64.0)
    ang = pos.to(torch.float64)[:, None] * theta
    c, s = torch.cos(ang).float()[:, None, :], torch.sin(ang).float()[:, None, :]
    a, b = x[..., :64], x[..., 64:]
    return torch.cat([a * c - b * s, b * c + a * s], dim=-1)


def _axis():
    """Axis of each of the 64 pairs: 16 turn with time, 24 with height, 24 with width."""
    return np.repeat(np.arange(3), [16, 24, 24]).astype(np.uint8)


def _positions(ctx, new):
    """[3][tokens]: the middle half of every chunk is an image 16 wide, the rest text."""
    out = []
    for s, n in zip(ctx, new):
        t = np.tile(np.arange(s - n, s), (3, 1))
        a, m = n // 4, n // 2
        at = np.arange(m)
        t[0, a:a + m] = t[0, a] if m else 0
        t[1, a:a + m] = t[0, a:a + m] + at // 16
        t[2, a:a + m] = t[0, a:a + m] + at % 16
        out.append(t)
    return np.concatenate(out, axis=1).astype(np.int32)


def _dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV, dtype)


def prepare(case, seed):
    case = dict(_DEFAULTS, **case)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    h, g, page, batch = case["h"], case["g"], case["page"], case["batch"]
    ctx, new = _lens(case)
    n = sum(new)
    pages = [-(-s // page) for s in ctx]
    pool, cols = sum(pages) + 3, max(pages)
    perm = torch.randperm(pool, generator=gen, device=DEV)
    k_pages = torch.randn((pool, g, page, D), generator=gen, device=DEV).to(dt)
    v_pages = torch.randn((pool, g, page, D), generator=gen, device=DEV).to(dt)
    table = torch.full((batch, cols), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, (s, p) in enumerate(zip(ctx, pages)):
        phys = perm[at:at + p]
        at += p
        table[b, :p] = phys.to(torch.int32)
        if case["op"] in ("attn", "weights"):
            rows = _rope(k_pages[phys].float().transpose(1, 2).reshape(p * page, g, D), torch.arange(p * page, device=DEV))
            k_pages[phys] = rows.view(p, page, g, D).transpose(1, 2).to(dt)
    cu = np.concatenate([[0], np.cumsum(new)])
    st = {"case": case, "k": k_pages, "v": v_pages, "table": table, "cu": _dev(cu), "cur": _dev(ctx), "ctx": ctx, "new": new}
    if case["op"] == "append":   # views of one fused projection
        qkv = torch.randn((n, (h + 2 * g) * D), generator=gen, device=DEV).to(dt)
        st["q"], st["kn"], st["vn"] = (t.view(n, -1, D) for t in torch.split(qkv, [h * D, g * D, g * D], dim=1))
        st["q_out"] = torch.zeros((n, h, D), dtype=dt, device=DEV)
        st["pos"] = _dev(_positions(ctx, new)) if case["axes"] > 1 else None
    elif case["op"] == "evict":  # weights as attention leaves them: over many orders of magnitude, some of them equal
        w = torch.exp(3.0 * torch.randn((batch, g, cols * page), generator=gen, device=DEV) - 8.0)
        w[:, :, ::7] = w[:, :, ::7].to(torch.bfloat16).float()
        st["w"], st["w_out"] = w, torch.zeros_like(w)
        st["ids"] = torch.zeros((batch, g, case["budget"]), dtype=torch.int32, device=DEV)
        st["kept"] = torch.zeros((batch,), dtype=torch.int32, device=DEV)
    else:
        pos = torch.cat([torch.arange(s - m, s, device=DEV) for s, m in zip(ctx, new)])
        st["q"] = _rope(2.0 * torch.randn((n, h, D), generator=gen, device=DEV), pos).to(dt)
        st["slopes"] = _dev(2.0 ** (-8.0 * np.arange(1, h + 1) / h), torch.float32) if case["bias"] else None
        st["first"] = _dev(np.concatenate([_first_key(case, s, m) for s, m in zip(ctx, new)])) if case["docs"] else None
        st["prefix"] = _dev(np.minimum(case["prefix"], ctx)) if case["prefix"] else None
        st["lse"] = torch.zeros((n, h), dtype=torch.float32, device=DEV)
        if case["op"] == "attn":
            st["out"] = torch.zeros((n, h, D), dtype=dt, device=DEV)
        else:
            for b, lo in enumerate(cu[:-1]):   # what the attention before it has returned
                for i in range(lo, cu[b + 1], 256):
                    j = min(i + 256, cu[b + 1])
                    z = _seq_scores(st, b, slice(i, j), torch.float32)
                    st["lse"][i:j] = torch.logsumexp(z, dim=-1).permute(2, 0, 1).reshape(j - i, h)
            st["w"] = torch.rand((batch, g, cols * page), generator=gen, device=DEV)
            st["w_out"] = torch.zeros_like(st["w"])
    if own:
        import paper_2512_15550_amd as ck
        st["cache"] = ck.ctkvr_cache_create(ck.CacheParams(
            batch=batch, n_q_heads=h, n_kv_heads=g, page_size=page, dtype=ck.BF16 if case["dtype"] == "bf16" else ck.F32, num_pages=pool,
            max_pages=cols, max_new=max(n, 1), softcap=case["cap"], rope_base=BASE, rope_axis=_axis() if case["axes"] > 1 else None))
    return st


# ------------------------------------------------------------------------------
# the plain forms
# ------------------------------------------------------------------------------
def _token(st):
    """Sequence and slot of every new token."""
    cu, cur = st["cu"].long(), st["cur"].long()
    t = torch.arange(st["q"].shape[0], device=DEV)
    b = torch.searchsorted(cu, t, right=True) - 1
    return b, cur[b] - cu[b + 1] + t


def _rows(pages, table):
    """The cache in order of tokens, [batch][g][slots][128] in 32 bits."""
    x = pages[table.long().clamp(min=0)].float()
    return x.transpose(1, 2).reshape(x.shape[0], x.shape[2], -1, D)


def _padded_scores(st):
    """Scores of a batch padded to its longest chunk, [batch][g][new][G][slots], and the tokens' places in it."""
    case = st["case"]
    g, group, n_max = case["g"], case["h"] // case["g"], max(st["new"])
    k = _rows(st["k"], st["table"])
    b, slot = _token(st)
    i = torch.arange(b.numel(), device=DEV) - st["cu"].long()[b]
    q = torch.zeros((len(st["new"]), n_max, g, group, D), device=DEV)
    q[b, i] = st["q"].float().view(-1, g, group, D)
    z = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(len(st["new"]), g, n_max * group, D), k.transpose(2, 3).contiguous())
    z = z.view(len(st["new"]), g, n_max, group, -1).mul_(1.0 / math.sqrt(D))
    if case["cap"]:
        z = z.div_(case["cap"]).tanh_().mul_(case["cap"])
    key = torch.arange(z.shape[-1], device=DEV)
    pos = torch.full((len(st["new"]), n_max), -1, dtype=torch.long, device=DEV)
    pos[b, i] = slot
    if st["slopes"] is not None:
        far = (pos[:, :, None] - key).abs().float()
        z -= st["slopes"].view(1, g, 1, group, 1) * far[:, None, :, None, :]
    seen = key <= pos[:, :, None]
    if st["prefix"] is not None:
        seen |= key < st["prefix"][:, None, None]
    if st["first"] is not None:
        first = torch.zeros_like(pos)
        first[b, i] = st["first"].long()
        seen &= key >= first[:, :, None]
    seen &= key < st["cur"][:, None, None]
    seen &= (pos >= 0)[:, :, None]
    return z.masked_fill_(~seen[:, None, :, None, :], -math.inf), b, i


def _attn(st):
    z, b, i = _padded_scores(st)
    m = z.amax(dim=-1, keepdim=True).clamp_(min=-1e30)
    p = z.sub_(m).exp_()
    l = p.sum(dim=-1, keepdim=True)
    bb, g, n_max, group, s = p.shape
    o = torch.matmul(p.view(bb, g, n_max * group, s), _rows(st["v"], st["table"])).view(bb, g, n_max, group, D) / l.clamp(min=1e-30)
    lse = torch.log(l) + m
    st["out"].copy_(o[b, :, i].reshape(st["out"].shape))
    st["lse"].copy_(lse[b, :, i].reshape(st["lse"].shape))
    return st["out"], st["lse"]


def _weights(st):
    z, b, i = _padded_scores(st)
    bb, g, n_max, group, s = z.shape
    lse = torch.zeros((bb, n_max, g, group), device=DEV)
    lse[b, i] = st["lse"].view(-1, g, group)
    w = z.sub_(lse.permute(0, 2, 1, 3)[..., None]).exp_().sum(dim=(2, 3))
    key = torch.arange(s, device=DEV)
    new = (st["cu"][1:] - st["cu"][:-1])[:, None]
    old = (key < st["cur"][:, None] - new)[:, None, :]
    w += torch.where(old, st["w"] * st["case"]["decay"], 0.0)
    st["w_out"].copy_(torch.where((key < st["cur"][:, None])[:, None, :], w, st["w_out"]))
    return st["w_out"]


def _append(st):
    case = st["case"]
    b, slot = _token(st)
    pos = st["pos"] if st["pos"] is not None else slot[None]
    axis = torch.from_numpy(_axis()).to(DEV).long() if case["axes"] > 1 else torch.zeros(64, dtype=torch.long, device=DEV)
    freq = BASE ** (-torch.arange(64, dtype=torch.float64, device=DEV) / 64.0)
    ang = pos[axis].to(torch.float64).transpose(0, 1) * freq      # (32 bits lose the angles of far positions)
    c, s = torch.cos(ang).float()[:, None, :], torch.sin(ang).float()[:, None, :]
    q, k = st["q"].float(), st["kn"].float()
    st["q_out"].copy_(torch.cat([q[..., :64] * c - q[..., 64:] * s, q[..., 64:] * c + q[..., :64] * s], dim=-1))
    k = torch.cat([k[..., :64] * c - k[..., 64:] * s, k[..., 64:] * c + k[..., :64] * s], dim=-1)
    page, at = st["table"][b, slot // case["page"]].long(), slot % case["page"]
    st["k"][page, :, at] = k.to(st["k"].dtype)
    st["v"][page, :, at] = st["vn"]
    return st["q_out"], st["k"], st["v"]


def _evict(st):
    case = st["case"]
    w, cur, budget = st["w"], st["cur"].long()[:, None, None], case["budget"]
    key = torch.arange(w.shape[-1], device=DEV)
    rank = torch.where((key < case["n_init"]) | (key >= cur - case["n_local"]), math.inf, w)
    rank = torch.where(key < cur, rank, -math.inf)
    order = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :budget]
    j = torch.arange(order.shape[-1], device=DEV)
    kept = j < cur.clamp(max=budget)
    ids = torch.sort(torch.where(kept, order, 1 << 30), dim=-1).values
    src = torch.where(kept, ids, j)                      # (the rest stay where they are)
    bb, g = w.shape[:2]
    b, kv = torch.arange(bb, device=DEV)[:, None, None], torch.arange(g, device=DEV)[None, :, None]
    table = st["table"].long().clamp(min=0)
    from_page, to_page = table[b, src // case["page"]], table[b, (j // case["page"])[None, None]]
    held = kept & (src != j)
    for pages in (st["k"], st["v"]):
        rows, at = pages[from_page, kv, src % case["page"]], held.nonzero(as_tuple=True)
        pages[to_page.expand_as(src)[at], at[1], at[2] % case["page"]] = rows[at]
    st["w_out"][..., :order.shape[-1]] = torch.where(kept, torch.gather(w, 2, src), st["w_out"][..., :order.shape[-1]])
    st["ids"].fill_(-1)
    st["ids"][..., :order.shape[-1]] = torch.where(kept, ids, -1).int()
    st["kept"].copy_(cur.view(-1).clamp(max=budget))
    return st["ids"], st["kept"], st["w_out"], st["k"], st["v"]


def run(st):
    op = st["case"]["op"]
    if own:
        import paper_2512_15550_amd as ck
        case, cache = st["case"], st["cache"]
        if op == "append":
            ck.ctkvr_cache_append(cache, st["q"], st["kn"], st["vn"], st["cu"], st["cur"], st["table"], st["q_out"], st["k"], st["v"],
                                  positions=st["pos"])
            return st["q_out"], st["k"], st["v"]
        if op == "attn":
            ck.ctkvr_cache_attn(cache, st["q"], st["k"], st["v"], st["cu"], st["cur"], st["table"], st["out"], out_lse=st["lse"],
                                slopes=st["slopes"], prefix_lens=st["prefix"], first_key=st["first"])
            return st["out"], st["lse"]
        if op == "weights":
            ck.ctkvr_cache_weights(cache, st["q"], st["lse"], st["k"], st["cu"], st["cur"], st["table"], st["w"], st["w_out"],
                                   decay=case["decay"], slopes=st["slopes"], prefix_lens=st["prefix"], first_key=st["first"])
            return st["w_out"]
        ck.ctkvr_cache_evict(cache, st["w"], st["k"], st["v"], st["cur"], st["table"], case["budget"], n_init=case["n_init"],
                             n_local=case["n_local"], weights_out=st["w_out"], out_ids=st["ids"], out_lens=st["kept"])
        return st["ids"], st["kept"], st["w_out"], st["k"], st["v"]
    return {"append": _append, "attn": _attn, "weights": _weights, "evict": _evict}[op](st)


# ------------------------------------------------------------------------------
# from the definitions in 64 bits, sequence by sequence
# ------------------------------------------------------------------------------
def _seq_scores(st, b, rows, dtype):
    """Scores of the tokens `rows` of sequence b, [g][G][rows][keys], -inf where a key is not visible."""
    case, s, n = st["case"], st["ctx"][b], st["new"][b]
    g, group = case["g"], case["h"] // case["g"]
    phys = st["table"][b, :-(-s // case["page"])].long()
    k = st["k"][phys].to(dtype).permute(1, 0, 2, 3).reshape(g, -1, D)[:, :s]
    q = st["q"][rows].to(dtype).view(-1, g, group, D).permute(1, 2, 0, 3)
    m = q.shape[2]
    z = torch.bmm(q.reshape(g, group * m, D), k.transpose(1, 2).contiguous()).view(g, group, m, s) / math.sqrt(D)
    if case["cap"]:
        z = case["cap"] * torch.tanh(z / case["cap"])
    first_row = int(st["cu"][b])
    pos = torch.arange(rows.start, rows.stop, device=DEV) - first_row + s - n
    key = torch.arange(s, device=DEV)
    if st["slopes"] is not None:
        z = z - st["slopes"].to(dtype).view(g, group, 1, 1) * (pos[:, None] - key).abs().to(dtype)
    hidden = (key > pos[:, None]) & (key >= (int(st["prefix"][b]) if st["prefix"] is not None else 0))
    if st["first"] is not None:
        hidden |= key < st["first"][rows].long()[:, None]
    return z.masked_fill(hidden, -math.inf)


def exact(case, seed):
    global own
    case, before = dict(_DEFAULTS, **case), own
    own = False
    try:
        st = prepare(case, seed)
    finally:
        own = before
    f8 = torch.float64
    ctx, new, g, h = st["ctx"], st["new"], case["g"], case["h"]
    cu = [0] + [int(x) for x in np.cumsum(new)]
    if case["op"] == "append":
        pos = _positions(ctx, new) if case["axes"] > 1 else np.concatenate([np.arange(s - n, s) for s, n in zip(ctx, new)])[None]
        axis = _axis() if case["axes"] > 1 else np.zeros(64, int)
        turn = torch.from_numpy(np.exp(1j * pos[axis].T * BASE ** (-np.arange(64) / 64.0))).to(DEV)[:, None, :]

        def rotated(x):
            y = torch.complex(x[..., :64].to(f8), x[..., 64:].to(f8)) * turn
            return torch.cat([y.real, y.imag], dim=-1)

        kk, vv, q, kn = st["k"].to(f8), st["v"].to(f8), rotated(st["q"]), rotated(st["kn"])
        for b, (s, n) in enumerate(zip(ctx, new)):
            t = torch.arange(s - n, s, device=DEV)
            phys, at = st["table"][b, t // case["page"]].long(), t % case["page"]
            kk[phys, :, at] = kn[cu[b]:cu[b + 1]]
            vv[phys, :, at] = st["vn"][cu[b]:cu[b + 1]].to(f8)
        return q, kk, vv
    if case["op"] == "evict":
        kk, vv, w_out = st["k"].to(f8), st["v"].to(f8), st["w_out"].to(f8)
        w_host = st["w"].cpu().numpy()
        for b, s in enumerate(ctx):
            m = min(s, case["budget"])
            if m == s:
                w_out[b, :, :m] = st["w"][b, :, :m].to(f8)
                continue
            for kv in range(g):
                mid = np.arange(case["n_init"], s - case["n_local"])
                best = mid[np.lexsort((mid, -w_host[b, kv, mid].astype(np.float64)))][:m - case["n_init"] - case["n_local"]]
                ids = torch.from_numpy(np.concatenate([np.arange(case["n_init"]), np.sort(best), np.arange(s - case["n_local"], s)])).to(DEV)
                j = torch.arange(m, device=DEV)
                src, dst = st["table"][b, ids // case["page"]].long(), st["table"][b, j // case["page"]].long()
                for out, pages in ((kk, st["k"]), (vv, st["v"])):
                    out[dst, kv, j % case["page"]] = pages[src, kv, ids % case["page"]].to(f8)
                w_out[b, kv, :m] = st["w"][b, kv, ids].to(f8)
        return None, None, w_out, kk, vv
    step = max(1, (1 << 28) // (h * max(ctx)))
    if case["op"] == "attn":
        out, lse = torch.zeros((sum(new), h, D), dtype=f8, device=DEV), torch.zeros((sum(new), h), dtype=f8, device=DEV)
    else:
        w = st["w_out"].to(f8)
    for b, (s, n) in enumerate(zip(ctx, new)):
        if case["op"] == "weights":
            w[b, :, :s] = 0.0
            w[b, :, :s - n] = case["decay"] * st["w"][b, :, :s - n].to(f8)
        else:
            v = st["v"][st["table"][b, :-(-s // case["page"])].long()].to(f8).permute(1, 0, 2, 3).reshape(g, -1, D)[:, :s].contiguous()
        for i in range(cu[b], cu[b + 1], step):
            rows = slice(i, min(i + step, cu[b + 1]))
            m = rows.stop - i
            z = _seq_scores(st, b, rows, f8)
            if case["op"] == "attn":
                lse[rows] = torch.logsumexp(z, dim=-1).permute(2, 0, 1).reshape(m, h)
                p = torch.softmax(z, dim=-1).nan_to_num(0.0).view(g, -1, s)
                out[rows] = torch.bmm(p, v).view(g, h // g, m, D).permute(2, 0, 1, 3).reshape(m, h, D)
            else:
                z = z - st["lse"][rows].to(f8).view(m, g, h // g).permute(1, 2, 0)[..., None]
                w[b, :, :s] += torch.exp(z).sum(dim=(1, 2))
    return (out, lse) if case["op"] == "attn" else w
