"""Plain 64-bit statements of the serving operators, on the CPU, and the
inputs that their tests share.  A token's cache is a list here; pages, tables
and tiles exist only where inputs are laid out."""
import math
import random

import torch

TINY = 2.0 ** -100


def quantize(x):
    """Codes and scales of rows, in binary64."""
    x = x.double()
    a = x.abs().amax(dim=1) if x.shape[1] else torch.zeros(x.shape[0], dtype=torch.float64)
    scale = torch.where(a < TINY, torch.zeros_like(a), a / 127.0)
    codes = torch.where(a[:, None] < TINY, torch.zeros_like(x), x * (127.0 / a)[:, None])
    return codes, scale


def product(a, sa, w, sw, bias=None):
    y = (a.double() @ w.double().t()) * sa.double()[:, None] * sw.double()[None]
    return y if bias is None else y + bias.double()


def rotate(x, cos, sin, positions):
    x = x.double().clone()
    if cos is None:
        return x
    h = cos.shape[1]
    c, s = cos.double()[positions.long()][:, None], sin.double()[positions.long()][:, None]
    a, b = x[..., :h].clone(), x[..., h:2 * h].clone()
    x[..., :h], x[..., h:2 * h] = a * c - b * s, b * c + a * s
    return x


def attend(q, k, v, first, scale, window=0):
    """q [n, heads, D] at positions first ..; k, v [tokens, kv heads, D]."""
    n, heads, D = q.shape
    kv = k.shape[1]
    out = torch.zeros(n, heads, D, dtype=torch.float64)
    for i in range(n):
        p = first + i
        lo = max(0, p - window + 1) if window else 0
        hi = min(p + 1, k.shape[0])
        if hi <= lo:
            continue
        for h in range(heads):
            g = h * kv // heads
            s = (k[lo:hi, g].double() @ q[i, h].double()) * scale
            out[i, h] = torch.softmax(s, 0) @ v[lo:hi, g].double()
    return out


class Paged:
    """A cache whose sequences lie in pages of a shuffled order: codes of
    about normal values, scales that differ from page to page, and in every
    place that no token holds codes of any value and scales that are not
    numbers."""

    def __init__(self, lengths, heads, D, page, seed, spare=3, spread=1.0, k_std=36.0):
        g = torch.Generator().manual_seed(seed)
        need = [-(-n // page) for n in lengths]
        self.n_pages = sum(need) + spare
        order = list(range(self.n_pages))
        random.Random(seed).shuffle(order)
        width = max(need + [1]) + 1
        self.table = torch.full((len(lengths), width), -7, dtype=torch.int32)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
            at += n
        draw = lambda *shape: (torch.randn(*shape, generator=g) * k_std).round().clamp(-127, 127).to(torch.int8)  # noqa: E731
        self.k = draw(self.n_pages, heads, page, D)
        self.v = draw(self.n_pages, heads, D, page)
        sc = lambda: torch.exp(spread * torch.randn(self.n_pages, heads, generator=g)) * (3.0 / 127.0)  # noqa: E731
        self.k_scale, self.v_scale = sc(), sc()
        for unused in order[at:]:
            self.k_scale[unused] = math.nan
            self.v_scale[unused] = math.inf
        self.lengths, self.page, self.heads, self.D = lengths, page, heads, D

    def slots(self, s, a, b):
        return [int(self.table[s, p // self.page]) * self.page + p % self.page for p in range(a, b)]

    def values(self, s, n=None):
        """(k, v) [tokens, heads, D] in binary64."""
        sl = torch.tensor(self.slots(s, 0, self.lengths[s] if n is None else n), dtype=torch.long)
        at, place = sl // self.page, sl % self.page
        k = self.k[at, :, place].double() * self.k_scale[at].double()[:, :, None]
        v = self.v[at, :, :, place].double() * self.v_scale[at].double()[:, :, None]
        return k, v

    def device(self, fs):
        t = lambda x: x.to("cuda:0")  # noqa: E731
        return fs.KVCache(t(self.k), t(self.v), t(self.k_scale), t(self.v_scale))


def attention_bound(q, k, v, first, scale, window, out, type_step):
    """How far a result may be from the 64-bit one, per element.

    The logits are off by at most e = 2^-11 * scale * max_j sum_d |q_d k_jd|
    (binary16 queries) or 2^-16 * scale * max|q| * max_j sum_d |k_jd| (15-bit
    queries), whichever path ran, plus 2^-20 of their size for binary32 sums;
    weights then by a factor e^(2e).  Probabilities are off by 2^-11 of
    themselves (binary16) or by 0.5 / 32512 of the largest of their 64 tokens,
    together at most 64 * 0.5 / 32512 of the weight.  Both move the result by
    no more than that share of the largest value; the store rounds by
    type_step of the result."""
    n, heads, D = q.shape
    kv = k.shape[1]
    bound = torch.zeros(n, heads, D, dtype=torch.float64)
    for h in range(heads):
        g = h * kv // heads
        if k.shape[0] == 0:
            break
        kk, qq = k[:, g].double().abs(), q[:, h].double().abs()
        size = (qq @ kk.t()).amax(dim=1) * scale
        e = torch.maximum(size * 2.0 ** -11, qq.amax(dim=1) * kk.sum(dim=1).max() * scale * 2.0 ** -16) + size * 2.0 ** -20
        share = torch.expm1(2 * e) + 64 * 0.5 / 32512
        bound[:, h] = share[:, None] * v[:, g].double().abs().amax()
    return bound + type_step * out.abs() + 1e-30
