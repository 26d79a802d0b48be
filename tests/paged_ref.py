"""Plain implementation of the paged 8-bit cache and the attention over it, used
by the GPU tests: the cache recipe of include/awsrc.h element by element on the
CPU (binary32 where the header fixes the rounding, 64 bits elsewhere), attention
in 64 bits."""
import math

import torch

E_MIN, E_MAX, E_NAN = -32, 31, -128


class Cache:
    """Codes as the values they stand for before their block's scale, [page, head, row, dim] in 64 bits."""

    def __init__(self, pages, heads, dim, page):
        self.pages, self.heads, self.dim, self.page = pages, heads, dim, page
        self.code = {w: torch.zeros(pages, heads, page, dim, dtype=torch.float64) for w in "kv"}
        self.exp = {w: torch.zeros(pages, heads, dtype=torch.int64) for w in "kv"}

    @staticmethod
    def of(dev):
        c = Cache(dev.pages, dev.kv_heads, dev.head_dim, dev.page)
        c.code["k"] = dev.k.cpu().double().permute(0, 1, 3, 2, 4).reshape(c.code["k"].shape)
        c.code["v"] = dev.v.cpu().double().permute(0, 1, 2, 4, 3).reshape(c.code["v"].shape)
        c.exp = {"k": dev.k_exp.cpu().long(), "v": dev.v_exp.cpu().long()}
        return c

    def values(self, which, pages, head, n):
        """The first n tokens of a sequence in these pages, [n, dim]."""
        e = self.exp[which][pages, head]
        s = torch.where(e == E_NAN, torch.nan, torch.exp2(e.double()))
        return (self.code[which][pages, head] * s[:, None, None]).reshape(-1, self.dim)[:n]


def e4m3(x):
    """Nearest e4m3 value, ties to even (64-bit arithmetic, |x| <= 448)."""
    _, p = torch.frexp(x)
    step = torch.exp2((p - 4).clamp(min=-9).double())
    return torch.round(x / step) * step


def exponent(amax):
    """Smallest e >= E_MIN with amax <= 448 * 2^e, by trying them."""
    if not (amax <= 448 * 2.0 ** E_MAX):
        return E_NAN
    e = E_MIN
    while amax > 448 * 2.0 ** e:
        e += 1
    return e


def rotate(x, cos, sin, interleaved):
    """x [tokens, heads, dim] float32; cos, sin [tokens, half] float32: every operation rounded to binary32."""
    h = cos.shape[1]
    y = x.clone()
    i = torch.arange(h)
    d1, d2 = (2 * i, 2 * i + 1) if interleaved else (i, i + h)
    c, s = cos[:, None], sin[:, None]
    y[..., d1] = x[..., d1] * c - x[..., d2] * s
    y[..., d2] = x[..., d2] * c + x[..., d1] * s
    return y


def append(cache, q, k, v, new, kv, table, cos, sin, interleaved):
    """Appends to `cache`; returns the rotated q in float32 (unrounded to q's dtype)."""
    pos = torch.cat([torch.arange(b - a, b) for a, b in zip(new, kv)])
    if cos is None:
        cos = sin = torch.zeros(int(pos.max()) + 1, 0)
    rows = {"k": rotate(k.float(), cos[pos], sin[pos], interleaved), "v": v.float()}
    P = cache.page
    for which, x in rows.items():
        at = 0
        for b, (n, total) in enumerate(zip(new, kv)):
            p = total - n
            while p < total:
                end = min(total, (p // P + 1) * P)
                pg, r = int(table[b][p // P]), p % P
                for h in range(cache.heads):
                    part = x[at:at + end - p, h]
                    need = exponent(float(part.abs().max())) if torch.isfinite(part).all() else E_NAN
                    old = int(cache.exp[which][pg, h]) if r else E_MIN
                    if E_NAN in (need, old):
                        e = E_NAN
                        cache.code[which][pg, h, r:r + end - p] = 0
                    else:
                        e = max(need, old)
                        if r:
                            cache.code[which][pg, h, :r] = e4m3(cache.code[which][pg, h, :r] * 2.0 ** (old - e))
                        cache.code[which][pg, h, r:r + end - p] = e4m3(part.double() * 2.0 ** -e)
                    cache.exp[which][pg, h] = e
                at, p = at + end - p, end
    return rotate(q.float(), cos[pos], sin[pos], interleaved)


def attention(cache, q, new, kv, table, scale, causal, eps_q, eps_p):
    """(out, lse, out bound, lse bound) in 64 bits. The bounds hold any computation that keeps q to a relative
    eps_q, the softmax weights to eps_p and sums in binary32:
      score error  d = scale sum|q k| (eps_q + (dim + 4) 2^-23) + 2^-22 |s| (its base-2 scaling and shift),
      weights      relative d + eps_p + 2^-21 (exp2), sums of n terms (n + 16) 2^-23,
    so |out - exact| <= 2 max_j(d + ...) sum_j p_j |v_j| and |lse - exact| <= the same relative error + 2^-22 |lse|."""
    n_tok, heads, dim = q.shape
    g = heads // cache.heads
    out = torch.zeros(n_tok, heads, dim, dtype=torch.float64)
    lse = torch.full((n_tok, heads), -math.inf, dtype=torch.float64)
    ob, lb = torch.zeros_like(out), torch.zeros_like(lse)
    at = 0
    for b, (n, total) in enumerate(zip(new, kv)):
        pages = [int(p) for p in table[b][:-(-total // cache.page)]]
        for h in range(heads if total and n else 0):
            k, v = (cache.values(w, pages, h // g, total) for w in "kv")
            x = q[at:at + n, h].double()
            s = x @ k.T * scale
            d = (x.abs() @ k.abs().T) * scale * (eps_q + (dim + 4) * 2.0 ** -23) + s.abs() * 2.0 ** -22
            if causal:
                hide = torch.arange(total)[None] > (total - n + torch.arange(n))[:, None]
                s, d = s.masked_fill(hide, -math.inf), d.masked_fill(hide, 0.0)
            rel = d.amax(1) + eps_p + 2.0 ** -21 + (total + 16) * 2.0 ** -23
            p = torch.softmax(s, 1)
            out[at:at + n, h] = p.nan_to_num(0) @ v if not torch.isnan(v).any() else p @ v
            lse[at:at + n, h] = torch.logsumexp(s, 1)
            ob[at:at + n, h] = 2 * rel[:, None] * (p @ v.abs())
            lb[at:at + n, h] = rel + lse[at:at + n, h].abs() * 2.0 ** -22
        at += n
    return out, lse, ob, lb
