"""Performance cases of decoding over a paged cache: what a server calls once per layer and step, over the sizes, data types and
options it calls it with, in plain torch and through the entry points of `paper_2510_22556_b200.binding`.

A case is a plain dict; `kind` names the operator:

  append   sablock_paged_append: rows of K and V go to their pages, keys and queries are rotated to their positions on the way, the
           bounds of the pages that they fall into (smallest and largest value of every channel of a page's keys) are kept up to date
  attend   sablock_paged_attention: the attention of one new token per sequence over all rows of its pages
  sparse   sablock_paged_sparse_attention: the same over the pages whose bounds promise the largest logits, chosen per KV head

A cache is a pool of pages k, v [n_pages, page, Hkv, D], a table [seqs, max_pages] of page numbers and the sequences' lengths,
all on the device.  Inputs are drawn from the seed alone: keys with a shared low-rank component (heavy-tailed logits), queries with a
common direction per KV head, pages in random order.
"""
from __future__ import annotations

import math
import random

import torch

own = False


def _case(**kw):
    c = dict(kind="attend", seqs=1, L=1024, L_min=0, new=1, new_min=0, len_seed=0, H=32, Hkv=8, D=128, dtype="bf16", page=64,
             rotary=0, interleaved=False, with_q=False, bounds=False, n_sel=0, n_first=1, n_last=1)
    c.update(kw)
    return c


def listed():
    return [
        # One token of one sequence, Llama-3-8B-shaped: the smallest call of a decoding loop, all latency.
        _case(name="append_one", kind="append", L=1057, rotary=128, with_q=True, bounds=True),
        # A step of a server batch: one token of each of 64 sequences behind their compacted prompts.
        _case(name="append_batch", kind="append", seqs=64, L=1500, L_min=1025, len_seed=1, page=32, rotary=128, with_q=True,
              bounds=True),
        # The prompts of five requests at once, ragged, behind what their caches hold already.
        _case(name="append_prompts", kind="append", seqs=5, L=5000, L_min=4097, len_seed=2, new=4000, new_min=300, rotary=128,
              with_q=True, bounds=True),
        # What the compression of 16 prompts retained moves into pages: no rotation, no queries.
        _case(name="append_compacted", kind="append", seqs=16, L=1024, L_min=1024, new=1024, new_min=1024, page=32, bounds=True),
        # The fp32 reference-sized model: one KV head, rotary pairs side by side on half of the channels, no bounds.
        _case(name="append_f32", kind="append", seqs=3, L=700, L_min=500, new=499, new_min=200, H=4, Hkv=1, D=64, dtype="f32",
              page=16, rotary=32, interleaved=True, with_q=True),
        # Decoding over one compacted prompt: the smallest attention.
        _case(name="attend_1k", L=1041),
        # The fp32 reference-sized model.
        _case(name="attend_f32", seqs=3, L=529, L_min=300, len_seed=5, H=4, Hkv=1, D=64, dtype="f32", page=16),
        # A server batch of compacted prompts.
        _case(name="attend_batch", seqs=64, L=1500, L_min=1025, len_seed=1, page=32),
        # 16 full prompts of 4K to 16K tokens.
        _case(name="attend_ragged16", seqs=16, L=16384, L_min=4096, len_seed=4),
        # One full prompt of 128K tokens.
        _case(name="attend_128k", L=131072),
        # The same prompt, 64 of its 2048 pages per KV head.
        _case(name="sparse_128k", kind="sparse", L=131072, bounds=True, n_sel=64),
        # 16 prompts of 4K to 16K tokens, 48 pages of 32 rows.
        _case(name="sparse_ragged16", kind="sparse", seqs=16, L=16384, L_min=4096, len_seed=4, page=32, bounds=True, n_sel=48),
    ]


def _log_uniform(rng: random.Random, lo: int, hi: int) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "sparse"])
    H, Hkv, D = rng.choice([(32, 8, 128), (32, 8, 128), (64, 8, 128), (32, 32, 128), (16, 8, 64), (8, 1, 128), (12, 2, 80), (8, 2, 256)])
    dtype = "f32" if rng.random() < 0.15 else "bf16"
    page = rng.choice([16, 32, 64, 64, 128])
    kw = dict(kind=kind, H=H, Hkv=Hkv, D=D, dtype=dtype, page=page, len_seed=rng.randint(0, 1 << 20))
    room = 131072 * 1024 // (Hkv * D * (2 if dtype == "f32" else 1))       # rows that are no more bytes than the largest listed case's
    if kind == "append":
        new = 1 if rng.random() < 0.4 else _log_uniform(rng, 2, 4000)
        seqs = _log_uniform(rng, 1, 64) if new == 1 else rng.randint(1, 8)
        new = max(1, min(new, room // 8 // seqs))
        L = new + _log_uniform(rng, 1, 1024)
        return _case(seqs=seqs, L=L + rng.randint(0, 200), L_min=L, new=new, new_min=max(1, new // 2), rotary=rng.choice([0, D, D, D // 2]),
                     interleaved=rng.random() < 0.3, with_q=rng.random() < 0.7, bounds=rng.random() < 0.6, **kw)
    L = _log_uniform(rng, 1 if kind == "attend" else 256, min(131072, room))
    seqs = max(1, min(_log_uniform(rng, 1, 64), room // L))
    kw.update(seqs=seqs, L=L, L_min=max(1, L // 3))
    if kind == "attend":
        return _case(**kw)
    return _case(bounds=True, n_sel=rng.choice([4, 16, 33, 64]), n_first=rng.choice([0, 1, 2]), n_last=rng.choice([1, 2]), **kw)


# ------------------------------------------------------------------------------------- sizes
def _lengths(c):
    """Rows of every sequence, the new ones among them, and how many are new."""
    r = random.Random(c["len_seed"])
    L = [r.randint(max(c["L_min"], 1), c["L"]) if c["seqs"] > 1 else c["L"] for _ in range(c["seqs"])]
    if c["kind"] != "append":
        return L, [0] * len(L)
    new = [r.randint(max(c["new_min"], 1), c["new"]) if c["seqs"] > 1 else c["new"] for _ in range(c["seqs"])]
    return [max(a, b) for a, b in zip(L, new)], new


def work(case):
    """Bytes: what is read and written once each, the bounds of the touched pages too.  Operations: rotations, logits and weighted
    values, and the scores of the pages."""
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    L, new = _lengths(c)
    row = c["Hkv"] * c["D"] * es
    pages = [-(-n // c["page"]) for n in L]
    if c["kind"] == "append":
        n, q = sum(new), c["H"] * c["D"] * es if c["with_q"] else 0
        touched = sum((a - 1) // c["page"] - (a - b) // c["page"] + 1 for a, b in zip(L, new))
        return {"bytes": n * (4 * row + 2 * q) + (4 * row * touched if c["bounds"] else 0),
                "flops": n * 3 * (c["rotary"] * c["Hkv"] + (c["rotary"] * c["H"] if c["with_q"] else 0)) + 1}
    io = len(L) * c["H"] * (c["D"] * (es + 4) + 4)
    if c["kind"] == "attend":
        return {"bytes": sum(L) * 2 * row + io, "flops": 4 * sum(L) * c["H"] * c["D"]}
    rows = sum(min(n, min(k, c["n_sel"]) * c["page"]) for n, k in zip(L, pages))
    return {"bytes": rows * 2 * row + sum(pages) * 2 * row + io, "flops": 4 * rows * c["H"] * c["D"] + 4 * sum(pages) * c["Hkv"] * c["D"]}


# ------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    L, new = _lengths(c)
    H, Hkv, D, ps, n = c["H"], c["Hkv"], c["D"], c["page"], len(L)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    max_pages = max(-(-x // ps) for x in L) + 1
    n_pages = n * max_pages
    mix = randn(8, Hkv, D) * (2 / math.sqrt(8))

    def keys(rows):
        return (randn(rows, Hkv, D) + torch.einsum("nr,rhd->nhd", randn(rows, 8), mix)).to(dt)

    lens = torch.tensor(L, dtype=torch.int32, device="cuda")
    table = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32).view(n, max_pages)
    k, v = (torch.empty(n_pages, ps, Hkv, D, dtype=dt, device="cuda") for _ in range(2))
    step = max(1, (1 << 26) // (ps * Hkv * D))
    for i in range(0, n_pages, step):
        m = min(step, n_pages - i)
        k[i:i + m] = keys(m * ps).view(m, ps, Hkv, D)
        v[i:i + m] = randn(m, ps, Hkv, D).to(dt)
    s = dict(case=c, k=k, v=v, lens=lens, table=table, bounds=None, handle=None)
    if c["bounds"]:
        # of the rows that are there before the call; pages without any hold what an earlier user of the page left
        old = (lens - torch.tensor(new, dtype=torch.int32, device="cuda")).long()
        fill = torch.full((n_pages,), ps, dtype=torch.int64, device="cuda")
        at = torch.arange(max_pages, device="cuda") * ps
        there = (old[:, None] - at[None]).clamp(0, ps)
        fill[table.view(-1).long()] = torch.where(there == 0, ps, there).view(-1)
        s["bounds"] = torch.empty(n_pages, Hkv, 2, D, dtype=dt, device="cuda")
        for i in range(0, n_pages, step):
            x = k[i:i + step].float()
            out = (torch.arange(ps, device="cuda")[None] >= fill[i:i + step, None])[:, :, None, None]
            s["bounds"][i:i + step, :, 0] = x.masked_fill(out, math.inf).amin(1).to(dt)
            s["bounds"][i:i + step, :, 1] = x.masked_fill(out, -math.inf).amax(1).to(dt)
    if c["kind"] != "append":
        s["q"] = (randn(n, H, D) + 1.5 * randn(n, Hkv, 1, D).expand(n, Hkv, H // Hkv, D).reshape(n, H, D)).to(dt)
        return s
    total = sum(new)
    s["cu"] = None
    if max(new) > 1:
        s["cu"] = torch.tensor([0] + new, device="cuda").cumsum(0).to(torch.int32)
    # one projection's output: queries, keys and values of a token side by side
    qkv = torch.cat([randn(total, H, D).to(dt), keys(total), randn(total, Hkv, D).to(dt)], 1)
    s["q"] = qkv[:, :H] if c["with_q"] else None
    s["new_k"], s["new_v"] = qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    # the positions go on from the prompt's, of which the cache holds only what was retained
    seq = torch.repeat_interleave(torch.arange(n, device="cuda"), torch.tensor(new, device="cuda"))
    first = torch.randint(0, 120000, (n,), generator=g, device="cuda")
    start = torch.tensor([0] + new[:-1], device="cuda").cumsum(0)
    s["positions"] = (first[seq] + torch.arange(total, device="cuda") - start[seq]).to(torch.int32)
    s["inv_freq"] = None
    if c["rotary"]:
        s["inv_freq"] = (500000.0 ** (-torch.arange(0, c["rotary"], 2, device="cuda", dtype=torch.float64) / c["rotary"])).float()
    return s


# ------------------------------------------------------------------------------------- plain forms
def _rotate(x, cos, sin, interleaved):
    """x [n, heads, D] in 32 bits, its first 2 * cos.shape[1] channels rotated in pairs."""
    half = cos.shape[1]
    cos, sin = cos[:, None], sin[:, None]
    r, rest = x[..., :2 * half], x[..., 2 * half:]
    if interleaved:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = r[..., :half], r[..., half:]
        r = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([r, rest], -1)


def _plain_append(s):
    c = s["case"]
    dt = s["k"].dtype
    t = torch.arange(s["new_k"].shape[0], device="cuda")
    if s["cu"] is None:
        seq, row = t, s["lens"].long() - 1
    else:
        cu = s["cu"].long()
        seq = torch.searchsorted(cu, t, right=True) - 1
        row = s["lens"].long()[seq] - cu[seq + 1] + t
    page, slot = s["table"][seq, row // c["page"]].long(), row % c["page"]
    q, k = s["q"], s["new_k"].float()
    if s["inv_freq"] is not None:
        angle = s["positions"].double()[:, None] * s["inv_freq"].double()[None]
        cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
        k = _rotate(k, cos, sin, c["interleaved"])
        q = None if q is None else _rotate(q.float(), cos, sin, c["interleaved"])
    k = k.to(dt)
    s["k"][page, slot], s["v"][page, slot] = k, s["new_v"]
    out = dict(k=s["k"], v=s["v"])
    if q is not None:
        out["q"] = q.to(dt)
    if s["bounds"] is not None:
        b = s["bounds"]
        fresh = slot == 0
        b[page[fresh], :, 0], b[page[fresh], :, 1] = k[fresh], k[fresh]
        b[:, :, 0] = b[:, :, 0].float().index_reduce(0, page, k.float(), "amin").to(dt)
        b[:, :, 1] = b[:, :, 1].float().index_reduce(0, page, k.float(), "amax").to(dt)
        out["bounds"] = b
    return out


def _weigh(q, k, v, seen):
    """q [n, Hkv, G, D]; k, v [n, Hkv, rows, D]; seen [n, 1 or Hkv, rows]: softmax(q k / sqrt D) v in 32 bits, and the log of the
    normaliser, both with the heads side by side."""
    x = (q @ k.transpose(-1, -2)) / math.sqrt(q.shape[-1])
    x = x.masked_fill(~seen[:, :, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    w = torch.exp(x - top)
    total = w.sum(-1, keepdim=True)
    return ((w @ v) / total).flatten(1, 2), (top + torch.log(total)).flatten(1)


def _plain_attend(s):
    c = s["case"]
    n, H, D = s["q"].shape
    k, v = (x[s["table"].long()].float().flatten(1, 2).transpose(1, 2) for x in (s["k"], s["v"]))
    seen = torch.arange(k.shape[2], device="cuda")[None, None] < s["lens"][:, None, None]
    out, lse = _weigh(s["q"].float().view(n, c["Hkv"], -1, D), k, v, seen)
    return dict(out=out, lse=lse)


def _plain_sparse(s):
    c = s["case"]
    n, H, D = s["q"].shape
    Hkv, ps, P = c["Hkv"], c["page"], s["table"].shape[1]
    table = s["table"].long()
    # scores next to the border decide which page is read: 64 bits, rounded once
    q = s["q"].double().view(n, Hkv, H // Hkv, D)
    b = s["bounds"][table].double()                                                   # [n, P, Hkv, 2, D]
    score = torch.einsum("nphd,nhd->nhp", b[:, :, :, 1], q.clamp(min=0).sum(2)) + torch.einsum("nphd,nhd->nhp", b[:, :, :, 0], q.clamp(max=0).sum(2))
    score = score.float()
    at = torch.arange(P, device="cuda")[None, None]
    pages = ((s["lens"].long() + ps - 1) // ps)[:, None, None]
    score = score.masked_fill((at < c["n_first"]) | (at >= pages - c["n_last"]), math.inf).masked_fill(at >= pages, -math.inf)
    best = torch.sort(score, dim=-1, descending=True, stable=True)[1][..., :c["n_sel"]]
    best = torch.nn.functional.pad(best, (0, c["n_sel"] - best.shape[-1]), value=P)
    best = torch.where(torch.arange(c["n_sel"], device="cuda") < pages, best, P).sort(-1)[0]   # ascending, absent ones last
    chosen = torch.where(best < P, best, -1)
    phys = table[torch.arange(n, device="cuda")[:, None, None], chosen.clamp(min=0)]
    head = torch.arange(Hkv, device="cuda")[None, :, None]
    k, v = (x.transpose(1, 2)[phys, head].float().flatten(2, 3) for x in (s["k"], s["v"]))      # [n, Hkv, n_sel * ps, D]
    row = (chosen[..., None] * ps + torch.arange(ps, device="cuda")).flatten(2)
    seen = (row >= 0) & (row < s["lens"][:, None, None]) & (chosen >= 0).repeat_interleave(ps, 2)
    out, lse = _weigh(s["q"].float().view(n, Hkv, -1, D), k, v, seen)
    return dict(out=out, lse=lse, selected=chosen.to(torch.int32))


def run(state):
    s = state
    c = s["case"]
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "sparse": _plain_sparse}[c["kind"]](s)
    from paper_2510_22556_b200 import binding as B
    if s["handle"] is None:            # the parameter block and the description of the cache, which a server makes once
        p = B.make_params(c["H"], c["Hkv"], c["D"], 1, s["k"].dtype)
        s["handle"] = p, B.make_pages(p, s["k"], s["v"], s["table"], s["lens"], s["bounds"])
    p, pages = s["handle"]
    if c["kind"] == "append":
        q = B.paged_append(p, pages, s["new_k"], s["new_v"], q=s["q"], positions=s["positions"], inv_freq=s["inv_freq"],
                           interleaved=c["interleaved"], cu_new=s["cu"])
        out = dict(k=s["k"], v=s["v"])
        if q is not None:
            out["q"] = q
        if s["bounds"] is not None:
            out["bounds"] = s["bounds"]
        return out
    if c["kind"] == "attend":
        out, lse = B.paged_attention(p, pages, s["q"], want_lse=True)
        return dict(out=out, lse=lse)
    out, selected, lse = B.paged_sparse_attention(p, pages, s["q"], c["n_sel"], n_first=c["n_first"], n_last=c["n_last"], want_lse=True)
    return dict(out=out, lse=lse, selected=selected)


# ------------------------------------------------------------------------------------- in 64 bits, from the definitions
def exact(case, seed):
    c = case
    s = prepare(case, seed)
    L, new = _lengths(c)
    ps, Hkv, G, D = c["page"], c["Hkv"], c["H"] // c["Hkv"], c["D"]
    if c["kind"] == "append":
        k, v = s["k"].double(), s["v"].double()
        bounds = None if s["bounds"] is None else s["bounds"].double()
        q_out = None if s["q"] is None else s["q"].double().clone()
        half, t0 = c["rotary"] // 2, 0

        def turn(x, z):
            """Pairs of channels as complex numbers, times z [n, half]."""
            y = x.double().clone()
            if half:
                i = torch.arange(half, device="cuda")
                a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + half)
                w = torch.complex(y[..., a], y[..., b]) * z[:, None]
                y[..., a], y[..., b] = w.real, w.imag
            return y

        for i, (length, n) in enumerate(zip(L, new)):
            new_k, new_v = s["new_k"][t0:t0 + n], s["new_v"][t0:t0 + n]
            z = None
            if half:
                phase = torch.outer(s["positions"][t0:t0 + n].double(), s["inv_freq"].double())
                z = torch.polar(torch.ones_like(phase), phase)
            rot = turn(new_k, z)
            if q_out is not None:
                q_out[t0:t0 + n] = turn(s["q"][t0:t0 + n], z)
            r0 = length - n
            for j in range(r0 // ps, (length - 1) // ps + 1):
                lo, hi = max(r0, j * ps), min(length, (j + 1) * ps)
                page = int(s["table"][i, j])
                part = rot[lo - r0:hi - r0]
                k[page, lo - j * ps:hi - j * ps] = part
                v[page, lo - j * ps:hi - j * ps] = new_v[lo - r0:hi - r0].double()
                if bounds is not None:
                    small, large = part.amin(0), part.amax(0)
                    if lo > j * ps:
                        small, large = torch.minimum(small, bounds[page, :, 0]), torch.maximum(large, bounds[page, :, 1])
                    bounds[page, :, 0], bounds[page, :, 1] = small, large
            t0 += n
        out = dict(k=k, v=v)
        if q_out is not None:
            out["q"] = q_out
        if bounds is not None:
            out["bounds"] = bounds
        return out
    res = torch.zeros(len(L), c["H"], D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(len(L), c["H"], dtype=torch.float64, device="cuda")
    for i, n in enumerate(L):
        for h in range(Hkv):
            q = s["q"][i, h * G:(h + 1) * G].double()
            pages = s["table"][i, :-(-n // ps)].long()
            rows = torch.arange(n, device="cuda")
            if c["kind"] == "sparse":
                b = s["bounds"][pages, h].double()
                score = torch.stack([torch.maximum(x * b[:, 0], x * b[:, 1]).sum(1) for x in q]).sum(0)
                m = len(pages)
                score[:c["n_first"]] = math.inf
                score[max(0, m - c["n_last"]):] = math.inf
                chosen = torch.topk(score, min(c["n_sel"], m))[1].sort()[0]
                rows = (chosen[:, None] * ps + torch.arange(ps, device="cuda")).flatten()
                rows = rows[rows < n]
            k, v = (x[pages[rows // ps], rows % ps, h].double() for x in (s["k"], s["v"]))
            x = q @ k.T / math.sqrt(D)
            res[i, h * G:(h + 1) * G] = torch.softmax(x, 1) @ v
            lse[i, h * G:(h + 1) * G] = torch.logsumexp(x, 1)
    return dict(out=res, lse=lse) if c["kind"] == "attend" else dict(out=res, lse=lse, selected=None)
