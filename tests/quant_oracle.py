"""Plain 64-bit implementations of the operators on a paged KV cache of 8-bit rows, in windows and for drafted tokens, on the CPU.  Written from the formulas of
include/ctkvr.h; nothing of the library is used."""
import math

import torch

from tests.cache_oracle import F8, HALF, Setup

TOP = {"int8": 127.0, "fp8": 448.0}
CODES = {"int8": torch.int8, "fp8": torch.float8_e4m3fn}


def half_step(y, store):
    """Half the distance between the codes around y, as the header has it: 1/2, or 2^-4 of y and 2^-10 at least."""
    return torch.full_like(y, 0.5) if store == "int8" else (y.abs() * 2.0 ** -4).clamp(min=2.0 ** -10)


def quantised(x, store):
    """Codes (their values in 64 bits) and scales of rows x [..., 128]: nearest codes of x * top / max |x|, ties to even; rows that are not finite: 0 and NaN."""
    x = x.to(F8)
    amax = x.abs().amax(dim=-1, keepdim=True)
    odd = ~torch.isfinite(x).all(dim=-1, keepdim=True)
    y = torch.where((amax > 0) & ~odd, x * TOP[store] / amax, 0.0)     # (x * top is exact, so that a tie is one)
    if store == "int8":
        codes = torch.round(y)
    else:
        e = torch.frexp(y.abs().clamp(min=2.0 ** -6)).exponent - 1
        step = torch.ldexp(torch.ones((), dtype=F8), e - 3)
        codes = torch.round(y / step) * step
    return codes, torch.where(odd, math.nan, amax / TOP[store]).squeeze(-1), y


class QuantSetup(Setup):
    """A Setup whose pages hold codes (k, v of the codes' type) and scales."""

    def __init__(self, seed, store, dtype, h, g, page, lens, new, **more):
        super().__init__(seed, dtype, h, g, page, lens, new, **more)
        self.store = store
        if store != "plain":
            for name in ("k", "v"):
                codes, scales, _ = quantised(getattr(self, name), store)
                setattr(self, name, codes.to(torch.float32).to(CODES[store]))
                setattr(self, name + "_scales", scales.float())
        else:
            self.k_scales = self.v_scales = None

    def held(self, name, b, kv, n):
        """The first n rows of a sequence's KV head in 64 bits, and which of them have a page."""
        t = torch.arange(n)
        page = self.table[b, t // self.page].long()
        ok = (page >= 0) & (page < self.num_pages)
        page, pages = page.clamp(0, self.num_pages - 1), getattr(self, name)
        if self.store == "plain":
            return pages[page, kv, t % self.page].to(F8), ok
        x = pages.view(torch.uint8)[page, kv, t % self.page].view(pages.dtype).float().to(F8)
        return x * getattr(self, name + "_scales")[page, kv, t % self.page].to(F8)[:, None], ok


def sees_range(st, b, prefix=None, first=None):
    s, n, c0 = st.lens[b], st.new[b], int(st.cu[b])
    pos, t = torch.arange(s - n, s)[:, None], torch.arange(s)[None, :]
    seen = t <= pos
    if prefix is not None:
        seen = seen | (t < int(prefix[b]))
    if first is not None:
        seen = seen & (t >= first[c0:c0 + n].long()[:, None])
    return seen


def sees_window(st, b, window, sinks):
    s, n = st.lens[b], st.new[b]
    pos, t = torch.arange(s - n, s)[:, None], torch.arange(s)[None, :]
    return (t <= pos) & ((t > pos - window) | (t < sinks))


def sees_tree(st, b, mask, first=None):
    s, n, c0 = st.lens[b], st.new[b], int(st.cu[b])
    t = torch.arange(s)[None, :]
    seen = (t < s - n).expand(n, s).clone()
    words = mask[c0:c0 + n].long() & 0xffffffff
    for j in range(min(n, 32 * mask.shape[1])):
        seen[:, s - n + j] = (words[:, j // 32] >> (j % 32) & 1).bool()
    if first is not None:
        seen &= t >= first[c0:c0 + n].long()[:, None]
    return seen


def attention(st, sees, cap=0.0, slopes=None, scale=1.0 / math.sqrt(128.0), spread=False):
    """out, lse and per-element bounds on a kernel's deviation.  sees(b): which key [len] each of b's new tokens sees.  spread: rows of values of very
    different sizes."""
    n_all, G = int(st.cu[-1]), st.h // st.g
    out, lse = torch.zeros((n_all, st.h, 128), dtype=F8), torch.full((n_all, st.h), -math.inf, dtype=F8)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(st.batch):
        n, s, c0 = st.new[b], st.lens[b], int(st.cu[b])
        if n == 0 or s == 0:
            continue
        seen = sees(b)
        pos, t = torch.arange(s - n, s)[:, None], torch.arange(s)[None, :]
        q = st.q[c0:c0 + n].to(F8).view(n, st.g, G, 128)
        for kv in range(st.g):
            k, ok = st.held("k", b, kv, s)
            v, _ = st.held("v", b, kv, s)
            vis = (seen & ok[None, :])[None].expand(G, n, s)
            any_row = vis.any(dim=0).any(dim=0)
            k, v = (torch.where(any_row[:, None], x, torch.zeros((), dtype=F8)) for x in (k, v))
            x = torch.matmul(q[:, kv].transpose(0, 1), k.T) * scale
            mag = torch.matmul(q[:, kv].transpose(0, 1).abs(), k.abs().T) * scale
            if cap:
                x = cap * torch.tanh(x / cap)
            if slopes is not None:
                far = slopes[kv * G:(kv + 1) * G].to(F8)[:, None, None] * (pos - t).abs().to(F8)
                x, mag = x - far, torch.maximum(mag, far)
            z = x.masked_fill(~vis, -math.inf)
            # sums of 128 products in fp32, of three parts each with fp32 queries, off by a step at most; a few more for the scales, cap, bias and exponent
            big = float(mag[vis].nan_to_num(0.0).max()) if vis.any() else 0.0
            err = big * (140 if st.dtype == "bf16" else 400) * 2.0 ** -23 + 2.0 ** -20 * (1.0 + cap)
            l = torch.logsumexp(z, dim=-1)
            p = torch.exp(z - l.clamp(min=-1e300)[..., None])
            o, size = torch.matmul(p, v), torch.matmul(p, v.abs())
            # probabilities off by exp(2 err), rounded to the type for the product (in bf16); its fp32 sum over s keys, of three parts each in fp32; the output's
            # own rounding
            rel = math.expm1(2 * err) + (HALF["bf16"] if st.dtype == "bf16" else 0.0) + ((1 if st.dtype == "bf16" else 3) * s + 16) * 2.0 ** -23
            rows = slice(kv * G, (kv + 1) * G)
            if spread:
                # weights are below 2^15 with a power of two above all scales as 2^11, so that probabilities may be up to 16 under a maximum that lags: fp16 ends at
                # 2^-25, 2^-36 of that power, which is twice the largest scale at most; and so for each of s keys
                size = size + (s * 2.0 ** -35 * v.abs().max()) / rel * (l.T[..., None].transpose(0, 1) > -math.inf)
            out[c0:c0 + n, rows] = o.transpose(0, 1)
            tol[c0:c0 + n, rows] = (size * rel + o.abs() * HALF[st.dtype] + 1e-30).transpose(0, 1)
            lse[c0:c0 + n, rows] = l.T
            tol_lse[c0:c0 + n, rows] = (err + s * 2.0 ** -23 + 2.0 ** -21 * (1 + l.clamp(min=-1e30).abs())).T
    return out, lse, tol, tol_lse


def tree(n, gen, branch=3, words=None):
    """A random tree of n drafted tokens: mask words int32 [n][words] and depths."""
    words = words or max(1, -(-n // 32))
    sees, depth = torch.zeros((n, 32 * words), dtype=torch.bool), [0] * n
    for i in range(n):
        parent = int(torch.randint(max(-1, i - branch), i, (1,), generator=gen)) if i else -1
        if parent >= 0:
            sees[i], depth[i] = sees[parent], depth[parent] + 1
        if i < 32 * words:
            sees[i, i] = True
    return words_of(sees), depth


def words_of(sees):
    """Rows of truth values (a multiple of 32) as int32 words, the first in the lowest bit."""
    w = (sees.view(sees.shape[0], -1, 32).long() << torch.arange(32)).sum(dim=-1)
    return torch.where(w >= 2 ** 31, w - 2 ** 32, w).int()
