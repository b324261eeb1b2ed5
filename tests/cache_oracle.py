"""Plain 64-bit implementations of the operators on the paged KV cache, on the CPU, and the inputs their tests share.  Written from the
formulas of include/ctkvr.h; nothing of the library is used."""
import math

import numpy as np
import torch

F8 = torch.float64
TD = {"bf16": torch.bfloat16, "f32": torch.float32}
#: half a step of a type, relative to the value
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


class Setup:
    """A paged cache of a ragged batch, on the CPU in its storage type.  lens: tokens in the cache; new: those of them that a call brings."""

    def __init__(self, seed, dtype, h, g, page, lens, new, spare_cols=1, behind=0, q_scale=1.0):
        r = torch.Generator().manual_seed(seed)
        self.dtype, self.h, self.g, self.page, self.lens, self.new = dtype, h, g, page, list(lens), list(new)
        self.td = TD[dtype]
        self.batch = len(lens)
        pages = [-(-s // page) for s in lens]
        self.cols = max(max(pages), 1) + spare_cols
        self.num_pages = sum(pages) + 2
        perm = torch.randperm(self.num_pages, generator=r)
        self.table = torch.full((self.batch, self.cols), -1, dtype=torch.int32)
        at = 0
        for b, p in enumerate(pages):
            self.table[b, :p] = perm[at:at + p].int()
            at += p
        self.k = torch.randn((self.num_pages, g, page, 128), generator=r).to(self.td)
        self.v = torch.randn((self.num_pages, g, page, 128), generator=r).to(self.td)
        self.cu = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32)
        self.cur = torch.tensor(lens, dtype=torch.int32)
        self.total = int(self.cu[-1]) + behind          # tokens behind the last sequence belong to none
        self.q = (q_scale * torch.randn((self.total, h, 128), generator=r)).to(self.td)
        self.gen = r

    def rows(self, pages, b, kv, n):
        """The first n rows of a sequence's KV head in 64 bits, and which of them have a page."""
        t = torch.arange(n)
        page = self.table[b, t // self.page].long()
        ok = (page >= 0) & (page < self.num_pages)
        return pages[page.clamp(0, self.num_pages - 1), kv, t % self.page].to(F8), ok


def scores(st, b, cap=0.0, slopes=None, prefix=None, first=None, scale=1.0 / math.sqrt(128.0)):
    """z [g][G][n][len] of sequence b with -inf where a key is not seen, and a bound on what fp32 sums make of q.k * scale."""
    s, n, G = st.lens[b], st.new[b], st.h // st.g
    c0 = int(st.cu[b])
    q = st.q[c0:c0 + n].to(F8).view(n, st.g, G, 128)
    pos, t = torch.arange(s - n, s)[:, None], torch.arange(s)[None, :]
    seen = t <= pos
    if prefix is not None:
        seen = seen | (t < int(prefix[b]))
    if first is not None:
        seen = seen & (t >= first[c0:c0 + n].long()[:, None])
    z = torch.empty((st.g, G, n, s), dtype=F8)
    big = torch.zeros((), dtype=F8)
    for kv in range(st.g):
        k, ok = st.rows(st.k, b, kv, s)
        vis = (seen & ok[None, :])[None].expand(G, n, s)
        x = torch.matmul(q[:, kv].transpose(0, 1), k.T) * scale
        mag = torch.matmul(q[:, kv].transpose(0, 1).abs(), k.abs().T) * scale
        if vis.any():
            big = torch.maximum(big, mag[vis].max())
        if cap:
            x = cap * torch.tanh(x / cap)
        if slopes is not None:
            x = x - slopes[kv * G:(kv + 1) * G].to(F8)[:, None, None] * (pos - t).abs().to(F8)
            if vis.any():
                big = torch.maximum(big, x[vis].abs().max())
        z[kv] = x.masked_fill(~vis, -math.inf)
    # 128 products and their sum in fp32, each off by a step at most (matrix cores may truncate); a few more for scale, cap, bias and exponent
    err = float(big) * 140 * 2.0 ** -23 + 2.0 ** -20 * (1.0 + cap)
    return z, err


def attention(st, **masks):
    """out, lse and per-element bounds on a kernel's deviation from them, for the tokens of the batch."""
    n_all, G = int(st.cu[-1]), st.h // st.g
    out, lse = torch.zeros((n_all, st.h, 128), dtype=F8), torch.full((n_all, st.h), -math.inf, dtype=F8)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(st.batch):
        n, s, c0 = st.new[b], st.lens[b], int(st.cu[b])
        if n == 0 or s == 0:
            continue
        z, err = scores(st, b, **masks)
        lse_b = torch.logsumexp(z, dim=-1)
        p = torch.exp(z - lse_b.clamp(min=-1e300)[..., None])
        for kv in range(st.g):
            v, _ = st.rows(st.v, b, kv, s)
            # a key that is not seen has no part in the sum, whatever its value
            seen_by_none = (p[kv] == 0).all(dim=0).all(dim=0)
            v = torch.where(seen_by_none[:, None], torch.zeros((), dtype=F8), v)
            o, size = torch.matmul(p[kv], v), torch.matmul(p[kv], v.abs())
            # probabilities off by exp(2 err), rounded to the type for the product; its fp32 sum over s keys; the output's own rounding
            rel = math.expm1(2 * err) + (HALF["bf16"] if st.dtype == "bf16" else 0.0) + (s + 8) * 2.0 ** -23
            out[c0:c0 + n, kv * G:(kv + 1) * G] = o.transpose(0, 1)
            tol[c0:c0 + n, kv * G:(kv + 1) * G] = (size * rel + o.abs() * HALF[st.dtype] + 1e-30).transpose(0, 1)
        lse[c0:c0 + n] = lse_b.permute(2, 0, 1).reshape(n, st.h)
        tol_lse[c0:c0 + n] = (err + s * 2.0 ** -23 + 2.0 ** -21 * (1 + lse_b.clamp(min=-1e30).abs())).permute(2, 0, 1).reshape(n, st.h)
    return out, lse, tol, tol_lse


def weights(st, lse, w_in, w_out, decay, **masks):
    """weights_out after the call (w_out: what it held before), and bounds."""
    got, tol = w_out.to(F8).clone(), torch.zeros_like(w_out, dtype=F8)
    for b in range(st.batch):
        n, s, c0 = st.new[b], st.lens[b], int(st.cu[b])
        w = torch.zeros((st.g, s), dtype=F8)
        if w_in is not None:
            w[:, :s - n] = decay * w_in[b, :, :s - n].to(F8)
        add, err = torch.zeros_like(w), 0.0
        if n and s:
            z, err = scores(st, b, **masks)
            l = lse[c0:c0 + n].to(F8).view(n, st.g, -1).permute(1, 2, 0)[..., None]
            add = torch.exp(z - l.clamp(min=-1e300)).masked_fill(l == -math.inf, 0.0).sum(dim=(1, 2))
            err += 2.0 ** -22 * (1 + float(l.clamp(min=-1e30)[l > -math.inf].abs().max()) if (l > -math.inf).any() else 1.0)
        rows = n * st.h // st.g
        got[b, :, :s] = w + add
        tol[b, :, :s] = add * (math.expm1(2 * err) + (rows + 64) * 2.0 ** -23) + (w.abs() + add) * 2.0 ** -23 + 1e-30
    return got, tol


def rotated(x, pos, freq, axis):
    """x [n][heads][128], pos [axes][n]: the rotated rows, and a bound for fp32 sine, cosine and products."""
    a = torch.tensor([[math.fmod(int(pos[axis[i], t]) * float(freq[i]), 2 * math.pi) for i in range(64)] for t in range(x.shape[0])], dtype=F8)
    c, s = torch.cos(a)[:, None], torch.sin(a)[:, None]
    u, w = x[..., :64].to(F8), x[..., 64:].to(F8)
    size = (u.abs() + w.abs()) * 2.0 ** -21
    return torch.cat([u * c - w * s, w * c + u * s], dim=-1), torch.cat([size, size], dim=-1)


def evicted(st, w, budget, n_init, n_local):
    """ids [batch][g][budget], lens, and the weights, K and V after the call (weights: zeros elsewhere)."""
    ids = np.full((st.batch, st.g, budget), -1, np.int32)
    lens = [min(s, budget) for s in st.lens]
    k, v, w_out = st.k.clone(), st.v.clone(), torch.zeros_like(w)
    for b, (s, m) in enumerate(zip(st.lens, lens)):
        for kv in range(st.g):
            if s <= budget:
                keep = np.arange(s)
            else:
                mid = np.arange(n_init, s - n_local)
                rank = np.where(np.isnan(w[b, kv, mid].numpy()), -math.inf, w[b, kv, mid].numpy().astype(np.float64) + 0.0)
                nan = np.isnan(w[b, kv, mid].numpy())
                order = np.lexsort((mid, nan, -rank))
                keep = np.concatenate([np.arange(n_init), np.sort(mid[order[:m - n_init - n_local]]), np.arange(s - n_local, s)])
            ids[b, kv, :m] = keep
            w_out[b, kv, :m] = w[b, kv, torch.from_numpy(keep).long()]
            for j, t in enumerate(keep):
                src, dst = int(st.table[b, t // st.page]), int(st.table[b, j // st.page])
                if 0 <= src < st.num_pages and 0 <= dst < st.num_pages:
                    k[dst, kv, j % st.page] = st.k[src, kv, t % st.page]
                    v[dst, kv, j % st.page] = st.v[src, kv, t % st.page]
    return ids, lens, w_out, k, v
