"""Plain references of the paged cache's operators in 64 bits (torch, row by row), and the caches that the tests use."""
import math

import torch

from paper_2510_22556_b200 import binding as B


class Cache:
    """Pools filled with NaN (whatever is not a row of a sequence must not be looked at), pages in random order, some of them nobody's."""

    def __init__(self, lens, Hkv, D, page, dtype, seed=0, spare=2, bounds=False, layout="rows", fill=float("nan"), max_pages=None):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.Hkv, self.D, self.page, self.dtype, self.n_seqs = Hkv, D, page, dtype, len(lens)
        self.max_pages = max_pages or max(1, max(-(-n // page) for n in lens) + 1)
        self.n_pages = self.n_seqs * self.max_pages + spare
        shape = (self.n_pages, page, Hkv, D)
        if layout == "rows":                       # [page][slot][head]
            self.k, self.v = (torch.full(shape, fill, dtype=dtype, device="cuda") for _ in range(2))
        elif layout == "heads":                    # [page][head][slot]
            self.k, self.v = (torch.full((self.n_pages, Hkv, page, D), fill, dtype=dtype, device="cuda").transpose(1, 2) for _ in range(2))
        else:                                      # K and V of a page side by side, of differing strides
            both = torch.full((self.n_pages, 2, page, Hkv, D), fill, dtype=dtype, device="cuda")
            self.k, self.v = both[:, 0], torch.full((self.n_pages, page, Hkv + 1, D), fill, dtype=dtype, device="cuda")[:, :, :Hkv]
        wide = torch.randperm(self.n_pages, generator=self.g, device="cuda")[: self.n_seqs * self.max_pages].to(torch.int32)
        self.table = torch.full((self.n_seqs, self.max_pages + 3), -7, dtype=torch.int32, device="cuda")[:, 1: self.max_pages + 1]
        self.table.copy_(wide.view(self.n_seqs, self.max_pages))
        self.bounds = torch.full((self.n_pages, Hkv, 2, D), fill, dtype=dtype, device="cuda") if bounds else None
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")

    def randn(self, *shape):
        return torch.randn(*shape, generator=self.g, device="cuda").to(self.dtype)

    def place(self, s, row):
        return int(self.table[s, row // self.page]), row % self.page

    def rows(self, s, n):
        """Index pair of the first n rows of sequence s."""
        r = torch.arange(n, device="cuda")
        return self.table[s, r // self.page].long(), r % self.page

    def fill(self):
        """Random rows for all sequences, and the bounds of their pages."""
        for s, n in enumerate(self.lens.tolist()):
            at = self.rows(s, n)
            self.k[at], self.v[at] = self.randn(n, self.Hkv, self.D), self.randn(n, self.Hkv, self.D)
            self.set_bounds(s, n)
        return self

    def set_bounds(self, s, n):
        if self.bounds is None:
            return
        for j in range(-(-n // self.page)):
            x = self.k[int(self.table[s, j]), : min(self.page, n - j * self.page)].float()
            self.bounds[int(self.table[s, j])] = torch.stack([x.amin(0), x.amax(0)], 1).to(self.dtype)

    def handle(self, p):
        return B.make_pages(p, self.k, self.v, self.table, self.lens, self.bounds)


def attend(q, k, v):
    """q [G, D], k, v [n, D]: attention and log-sum-exp in 64 bits."""
    if k.shape[0] == 0:
        return torch.zeros(q.shape, dtype=torch.float64, device=q.device), torch.full((q.shape[0],), -math.inf, dtype=torch.float64, device=q.device)
    x = q.double() @ k.double().T / math.sqrt(q.shape[1])
    return torch.softmax(x, 1) @ v.double(), torch.logsumexp(x, 1)


def attention(c, q, selected=None, absent=()):
    """Over all rows, or the pages selected [n_seqs][Hkv] lists; `absent`: pages (sequence, index) that are not there."""
    n, H, D = q.shape
    G = H // c.Hkv
    out = torch.zeros(n, H, D, dtype=torch.float64, device=q.device)
    lse = torch.zeros(n, H, dtype=torch.float64, device=q.device)
    for s, length in enumerate(c.lens.tolist()):
        length = min(max(length, 0), c.max_pages * c.page)
        for h in range(c.Hkv):
            r = torch.arange(length, device="cuda")
            if selected is not None:
                r = torch.cat([torch.arange(j * c.page, min((j + 1) * c.page, length), device="cuda") for j in selected[s][h]] + [r[:0]])
            for t, j in absent:
                if t == s:
                    r = r[r // c.page != j]
            at = c.table[s, r // c.page].long(), r % c.page, torch.full_like(r, h)
            g = slice(h * G, (h + 1) * G)
            out[s, g], lse[s, g] = attend(q[s, g], c.k[at], c.v[at])
    return out, lse


def scores(c, q):
    """[n_seqs][Hkv][pages] in 64 bits, rounded to 32."""
    n, H, D = q.shape
    G = H // c.Hkv
    res = []
    for s, length in enumerate(c.lens.tolist()):
        pages = c.table[s, : -(-length // c.page)].long()
        b = c.bounds[pages].double()
        x = q[s].double().view(c.Hkv, G, D)
        res.append([sum(torch.maximum(x[h, i] * b[:, h, 0], x[h, i] * b[:, h, 1]).sum(1) for i in range(G)).float() for h in range(c.Hkv)])
    return res


def choose(score, n_sel, n_first, n_last):
    """Pages chosen from one list of scores, ascending."""
    n = score.numel()
    forced = set(range(min(n_first, n))) | set(range(max(0, n - n_last), n))
    if n <= n_sel:
        return list(range(n))
    x = score.tolist()
    rest = sorted((j for j in range(n) if j not in forced), key=lambda j: (not math.isnan(x[j]), -x[j] if not math.isnan(x[j]) else 0, j))
    return sorted(list(forced) + rest[: n_sel - len(forced)])


def rotate(x, positions, inv_freq, interleaved):
    """x [n, heads, D] in 64 bits."""
    x = x.double().clone()
    if inv_freq is None:
        return x
    half = inv_freq.numel()
    angle = positions.double()[:, None, None] * inv_freq.double()
    i = torch.arange(half, device=x.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    u, w = x[..., a].clone(), x[..., b].clone()
    x[..., a], x[..., b] = u * angle.cos() - w * angle.sin(), w * angle.cos() + u * angle.sin()
    return x
