"""The paged cache on the GPU against plain references in 64 bits: appending with rotation and bounds, attention over all rows, choice
of pages, attention over chosen pages, and all of them behind a compression as a decoder runs them.

Tolerances.  Appending: a rounding to the cache's type is off by at most half a step (bf16 2^-8 of the value; none of its own in fp32),
the rotation in fp32 by 2^-20 (|x| + |y|) of the pair (angle to 2^-24 turns, sine and cosine to 2 ulp, two products and a sum).
Attention: a logit is an fp32 sum of D <= 256 products, partial sums below 16, so off by about sqrt(256) 2^-24 16 = 1.5e-5, which is the
relative error of a weight; an output is a convex combination of rows of V: 2e-5 max |V|, a log-sum-exp 1e-4."""
import math

import pytest
import torch

import paged_reference as R
import synth
from paged_reference import Cache
from paper_2510_22556_b200 import binding as B
from paper_2510_22556_b200 import build as build_lib

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_lib()
    B.lib()


def _params(H, Hkv, D, dtype):
    return B.make_params(H, Hkv, D, 1, dtype)


# ------------------------------------------------------------------------------------------ appending
def _near(got, ref, pair, dtype):
    """|got - ref| within a rounding and the rotation's error; pair: |x| + |y|."""
    lim = 2.0 ** -20 * pair + (2.0 ** -8 * ref.abs() if dtype == BF16 else 0)
    assert bool(((got.double() - ref).abs() <= lim).all()), float(((got.double() - ref).abs() - lim).max())


@pytest.mark.parametrize("H,Hkv,D,dtype,rotary,interleaved", [
    (32, 8, 128, BF16, 128, False), (8, 8, 64, BF16, 64, True), (6, 2, 80, BF16, 40, False), (6, 2, 80, BF16, 80, False), (4, 1, 256, BF16, 64, False),
    (3, 3, 96, BF16, 0, False), (4, 1, 64, F32, 64, False), (8, 2, 128, F32, 32, True), (2, 2, 20, F32, 12, False), (2, 1, 256, F32, 256, False),
    (2, 1, 8, BF16, 2, False), (40, 40, 128, BF16, 128, False)])
@pytest.mark.parametrize("page,new,old,layout", [
    (16, None, [0, 15, 16, 40, 31], "rows"),              # one token each: first of all, last of a page, first of a page
    (16, [1, 0, 17, 33, 5], [0, 9, 15, 16, 3], "heads"),
    (1, [3, 2, 1, 0, 4], [0, 1, 5, 2, 0], "rows"),
    (20, [70, 1, 20, 0, 23], [13, 19, 0, 4, 37], "both"),
    (64, [130, 64, 1, 0, 200], [0, 0, 63, 5, 31], "rows")])
@pytest.mark.parametrize("bounds", [False, True])
def test_append(H, Hkv, D, dtype, rotary, interleaved, page, new, old, layout, bounds):
    n_new = new or [1] * len(old)
    total, pad = sum(n_new), 2 if new else 0
    c = Cache([a + b for a, b in zip(old, n_new)], Hkv, D, page, dtype, seed=D + page, bounds=bounds, layout=layout)
    for s, n in enumerate(old):                            # the rows that are there
        at = c.rows(s, n)
        c.k[at], c.v[at] = c.randn(n, Hkv, D), c.randn(n, Hkv, D)
        c.set_bounds(s, n)
    qkv = c.randn(total + pad, H + 2 * Hkv, D)             # one projection's output, padded behind the last sequence
    q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    pos = torch.randint(0, 200000, (total + pad,), generator=c.g, device="cuda", dtype=torch.int32)
    freq = (10000.0 ** (-torch.arange(0, rotary, 2, device="cuda", dtype=torch.float64) / rotary)).float() if rotary else None
    cu = torch.tensor([0] + n_new, device="cuda").cumsum(0).to(torch.int32) if new else None
    k0, v0, b0 = c.k.clone(), c.v.clone(), None if c.bounds is None else c.bounds.clone()
    q_out = torch.full((total + pad, H, D), 7.0, dtype=dtype, device="cuda")
    p = _params(H, Hkv, D, dtype)
    assert B.paged_append(p, c.handle(p), k, v, q=q, positions=pos, inv_freq=freq, interleaved=interleaved, cu_new=cu, q_out=q_out) is q_out
    assert B.last_launch_count() == (2 if bounds and new and page > 32 else 1)
    size = R.rotate(qkv.abs(), torch.zeros_like(pos), freq, interleaved)
    if rotary:
        i = torch.arange(rotary // 2, device="cuda")
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)
        size[..., a] = size[..., b] = size[..., a] + size[..., b]
    ref = R.rotate(qkv, pos, freq, interleaved)
    _near(q_out[:total], ref[:total, :H], size[:total, :H], dtype)
    assert bool((q_out[total:] == 7).all())
    t = 0
    for s, n in enumerate(n_new):
        for r in range(old[s], old[s] + n):
            at = c.place(s, r)
            _near(c.k[at], ref[t, H:H + Hkv], size[t, H:H + Hkv], dtype)
            assert torch.equal(c.v[at], v[t])
            k0[at], v0[at] = c.k[at], c.v[at]
            t += 1
    assert torch.equal(c.k.nan_to_num(9e9), k0.nan_to_num(9e9)) and torch.equal(c.v.nan_to_num(9e9), v0.nan_to_num(9e9))      # nothing else was written
    if bounds:
        got = c.bounds.clone()
        c.bounds.copy_(b0)
        for s, n in enumerate(n_new):
            if n:
                c.set_bounds(s, old[s] + n)
        assert torch.equal(got.nan_to_num(9e9), c.bounds.nan_to_num(9e9))


def test_append_far_positions_and_row_positions():
    """Angles of positions near 2^31, and positions taken from the rows."""
    c = Cache([300], 2, 64, 16, F32)
    p = _params(2, 2, 64, F32)
    freq = (10000.0 ** (-torch.arange(0, 64, 2, device="cuda", dtype=torch.float64) / 64)).float()
    k = c.randn(300, 2, 64)
    cu = torch.tensor([0, 300], dtype=torch.int32, device="cuda")
    for pos in (torch.arange(2 ** 31 - 300, 2 ** 31, device="cuda").to(torch.int32), None):
        B.paged_append(p, c.handle(p), k, k, positions=pos, inv_freq=freq, cu_new=cu)
        ref = R.rotate(k, torch.arange(300, device="cuda") if pos is None else pos, freq, False)
        # turns are formed in double: at 2^31 they are off by 2^-53 2^31 = 2^-22, an angle by 2 pi times that
        assert float((c.k[c.rows(0, 300)].double() - ref).abs().max()) <= 2.0 ** -18 * float(k.abs().max())


def test_append_does_not_follow_what_cannot_be():
    """Page numbers outside the pool, lengths below zero and above the table, sequences shorter than their new tokens, offsets that
    run backwards: what has a place is written, nothing else is."""
    p = _params(4, 2, 64, BF16)
    c = Cache([5, 5, 5, 5, 5, 5], 2, 64, 4, BF16, fill=1.0, max_pages=2, bounds=True)
    c.table[0, 1], c.table[1, 1] = -1, c.n_pages
    c.lens.copy_(torch.tensor([5, 5, -3, 9, 2, 5]))
    cu = torch.tensor([0, 2, 4, 6, 8, 11, 10], dtype=torch.int32, device="cuda")
    k, v, q = c.randn(12, 2, 64), c.randn(12, 2, 64), c.randn(12, 4, 64)
    k0, q_out = c.k.clone(), torch.full((12, 4, 64), 7.0, dtype=BF16, device="cuda")
    B.paged_append(p, c.handle(p), k, v, q=q, cu_new=cu, q_out=q_out)
    for s, row, t in [(0, 3, 0), (1, 3, 2), (3, 7, 6), (4, 0, 9), (4, 1, 10)]:      # sequence 3: row 8 is behind its table
        k0[c.place(s, row)] = k[t]
        assert torch.equal(q_out[t], q[t])
    assert torch.equal(c.k, k0)
    none = [1, 3, 4, 5, 7, 8, 11]
    assert bool((q_out[none] == 7).all())


def test_append_bounds_keep_what_is_no_number():
    p = _params(2, 1, 16, F32)
    c = Cache([6], 1, 16, 8, F32, bounds=True)
    k = c.randn(6, 1, 16)
    k[2, 0, 3], k[4, 0, 5], k[1, 0, 7] = float("nan"), float("inf"), -float("inf")
    B.paged_append(p, c.handle(p), k, k, cu_new=torch.tensor([0, 6], dtype=torch.int32, device="cuda"))
    lo, hi = c.bounds[int(c.table[0, 0]), 0]
    assert torch.equal(lo.isnan().nonzero().flatten().cpu(), torch.tensor([3])) and torch.equal(lo.isnan(), hi.isnan())
    assert float(hi[5]) == math.inf and float(lo[7]) == -math.inf


# ------------------------------------------------------------------------------------------ attention
SHAPES = [(32, 8, 128, BF16), (8, 1, 128, BF16), (5, 1, 128, BF16), (12, 1, 128, BF16), (40, 2, 64, BF16), (8, 8, 64, BF16), (6, 2, 80, BF16),
          (8, 2, 256, BF16), (12, 1, 192, BF16), (7, 7, 8, BF16), (34, 2, 128, BF16), (4, 1, 64, F32), (8, 1, 128, F32), (6, 3, 20, F32), (9, 1, 256, F32)]
LENS = [0, 1, 15, 16, 17, 33, 64, 65, 500, 1]


def _check_attention(c, p, q, selected=None, lists=None, absent=(), scale=1.0, call=None):
    """The call (attention over all rows or the pages `selected`, unless another one is given) against the reference."""
    ref, ref_lse = R.attention(c, q, lists, absent)
    g = c.handle(p)
    call = call or (lambda: B.paged_attention(p, g, q, selected=selected, want_lse=True))
    out, lse = call()
    top = max([float(c.v[c.rows(s, min(max(n, 0), c.max_pages * c.page))].double().abs().max()) for s, n in enumerate(c.lens.tolist()) if n > 0] or [1.0]) \
        if not absent else float(c.v.double().nan_to_num(0).abs().max())
    assert float((out.double() - ref).abs().max()) <= 2e-5 * scale * top
    empty = ref_lse == -math.inf
    assert torch.equal(empty, lse == -math.inf)
    assert bool((out[empty] == 0).all())
    if not bool(empty.all()):
        assert float((lse.double() - ref_lse)[~empty].abs().max()) <= 1e-4 * scale
    assert torch.equal(out, call()[0])                                             # fixed order


@pytest.mark.parametrize("H,Hkv,D,dtype", SHAPES)
@pytest.mark.parametrize("page,layout", [(16, "rows"), (1, "heads"), (20, "both"), (128, "rows")])
def test_attention(H, Hkv, D, dtype, page, layout):
    c = Cache(LENS, Hkv, D, page, dtype, seed=D * page, layout=layout).fill()
    q = (c.randn(len(LENS), H, D).float() * 1.5).to(dtype)
    _check_attention(c, _params(H, Hkv, D, dtype), q)


@pytest.mark.parametrize("H,Hkv,D,dtype", [(32, 8, 128, BF16), (8, 1, 128, BF16), (12, 1, 64, BF16), (4, 1, 256, BF16), (4, 1, 64, F32), (8, 1, 256, F32)])
@pytest.mark.parametrize("lens", [[1], [64], [1041], [9000], [30000, 7, 0, 12345], [0], [0, 0], [200] * 70, [3] * 600])
def test_attention_shares(H, Hkv, D, dtype, lens):
    """Pairs cut by the shares of many CTAs, shares of many pairs, fewer units than CTAs."""
    c = Cache(lens, Hkv, D, 64, dtype, seed=len(lens), fill=0.0).fill()
    q = (c.randn(len(lens), H, D).float() * 1.5).to(dtype)
    if max(lens) > 500:
        c.k[c.place(0, lens[0] // 2)] *= 12                # a late logit far above the first ones
    _check_attention(c, _params(H, Hkv, D, dtype), q, scale=12)


def test_attention_many_sequences():
    """More sequences than the threads that add their lengths up."""
    lens = [(i * 7) % 41 for i in range(1000)]
    c = Cache(lens, 1, 64, 16, BF16, fill=0.0).fill()
    _check_attention(c, _params(2, 1, 64, BF16), c.randn(1000, 2, 64))


def test_attention_offsets_past_32_bits():
    """A pool of more than 2^32 elements, the rows in its last pages."""
    n_pages, page, Hkv, D = 2200, 2048, 8, 128                      # 4.6e9 elements, 9.2 GB each
    k, v = (torch.empty(n_pages, page, Hkv, D, dtype=BF16, device="cuda") for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(3)
    used = [2199, 2150, 2101]
    for x in (k, v):
        for j in used:
            x[j] = torch.randn(page, Hkv, D, generator=g, device="cuda").to(BF16)
    table = torch.tensor([used], dtype=torch.int32, device="cuda")
    lens = torch.tensor([5000], dtype=torch.int32, device="cuda")
    p = _params(32, 8, 128, BF16)
    pages = B.make_pages(p, k, v, table, lens)
    q = torch.randn(1, 32, 128, generator=g, device="cuda").to(BF16)
    out = B.paged_attention(p, pages, q)
    kk, vv = (torch.cat([x[j] for j in used])[:5000] for x in (k, v))
    for h in range(8):
        ref, _ = R.attend(q[0, 4 * h:4 * h + 4], kk[:, h], vv[:, h])
        assert float((out[0, 4 * h:4 * h + 4].double() - ref).abs().max()) <= 2e-5 * float(vv.float().abs().max())
    new = torch.randn(1, 8, 128, generator=g, device="cuda").to(BF16)
    lens += 1
    B.paged_append(p, pages, new, new)
    assert torch.equal(k[2101, 5000 - 4096], new[0])
    del k, v, pages
    torch.cuda.empty_cache()


def test_attention_does_not_follow_what_cannot_be():
    for H, Hkv, D, dtype in [(8, 2, 128, BF16), (4, 1, 64, F32)]:
        c = Cache([50, 50, 50, 50], Hkv, D, 8, dtype, max_pages=7).fill()
        c.table[0, 2], c.table[0, 6], c.table[1, 0] = -1, c.n_pages, -2 ** 31
        c.table[2] = 2 ** 31 - 1
        c.lens.copy_(torch.tensor([50, 50, 50, -4]))
        q = c.randn(4, H, D)
        absent = [(0, 2), (0, 6), (1, 0)] + [(2, j) for j in range(7)]
        _check_attention(c, _params(H, Hkv, D, dtype), q, absent=absent)
        c = Cache([56], Hkv, D, 8, dtype, max_pages=7).fill()          # a length above what the table holds counts as that
        q = c.randn(1, H, D)
        p = _params(H, Hkv, D, dtype)
        ref = B.paged_attention(p, c.handle(p), q)
        c.lens.fill_(1000)
        assert torch.equal(ref, B.paged_attention(p, c.handle(p), q))


@pytest.mark.parametrize("H,Hkv,D,dtype", [(8, 2, 128, BF16), (8, 1, 128, BF16), (16, 1, 64, BF16), (4, 2, 256, BF16), (4, 1, 64, F32)])
def test_attention_infinite_and_missing_values(H, Hkv, D, dtype):
    """An infinity in V stays one, of its sign, in its column; no number in a key or value of a row makes none of what sees it; rows that
    are not the sequence's may hold anything (the pools are full of NaN)."""
    c = Cache([700, 700, 300], Hkv, D, 32, dtype, seed=D).fill()
    q = c.randn(3, H, D)
    for row, col, x in ((5, 3, math.inf), (350, 5, -math.inf), (699, 7, math.inf)):
        c.v[c.place(0, row)][:, col] = x
    c.v[c.place(1, 130)][:, 2] = float("nan")
    c.k[c.place(2, 299)][0] = float("nan")
    p = _params(H, Hkv, D, dtype)
    ref, _ = R.attention(c, q)
    out = B.paged_attention(p, c.handle(p), q).double()
    assert torch.equal(ref.isnan(), out.isnan()) and torch.equal(ref.isinf(), out.isinf())
    assert bool((out[ref.isinf()] == ref[ref.isinf()]).all())
    fin = ref.isfinite()
    assert float((out - ref)[fin].abs().max()) <= 2e-5 * 6


# ------------------------------------------------------------------------------------------ choosing pages
@pytest.mark.parametrize("H,Hkv,D,dtype", [(32, 8, 128, BF16), (8, 1, 64, BF16), (6, 2, 80, BF16), (4, 2, 256, BF16), (4, 1, 64, F32), (6, 1, 256, F32),
                                           (2, 2, 128, F32), (3, 1, 8, BF16)])
@pytest.mark.parametrize("page,lens,n_sel,n_first,n_last", [
    (16, [0, 1, 64, 65, 900, 1000], 4, 1, 1), (4, [4000, 13, 12, 2222], 64, 2, 3), (1, [9000, 5], 33, 0, 0), (32, [5000], 1, 0, 1), (16, [3000, 40], 7, 7, 0)])
def test_page_select_and_attention_over_it(H, Hkv, D, dtype, page, lens, n_sel, n_first, n_last):
    c = Cache(lens, Hkv, D, page, dtype, seed=page + D, bounds=True).fill()
    q = c.randn(len(lens), H, D)
    p = _params(H, Hkv, D, dtype)
    g = c.handle(p)
    want = [[R.choose(x, n_sel, n_first, n_last) for x in heads] for heads in R.scores(c, q)]
    sel = B.page_select(p, g, q, n_sel, n_first, n_last)
    assert sel.tolist() == [[x + [-1] * (n_sel - len(x)) for x in heads] for heads in want]
    _check_attention(c, p, q, sel, want)

    def both():
        out, chosen, lse = B.paged_sparse_attention(p, g, q, n_sel, n_first, n_last, want_lse=True)
        assert torch.equal(chosen, sel)
        return out, lse
    _check_attention(c, p, q, None, want, call=both)


def test_page_select_ties_infinities_and_missing_numbers():
    p = _params(2, 1, 16, F32)
    c = Cache([4 * 300], 1, 16, 4, F32, bounds=True).fill()
    q = c.randn(1, 2, 16)
    pages = c.table[0, :300].long()
    c.bounds[pages] = c.bounds[pages[0]].clone()                      # all the same: the lowest come in
    assert B.page_select(p, c.handle(p), q, 5, 0, 0).tolist() == [[[0, 1, 2, 3, 4]]]
    assert B.page_select(p, c.handle(p), q, 5, 0, 1).tolist() == [[[0, 1, 2, 3, 299]]]
    assert B.page_select(p, c.handle(p), q, 299, 0, 0).tolist() == [[list(range(299))]]
    c.bounds[pages[200], 0, 1] += 1.0
    c.bounds[pages[200], 0, 0] -= 1.0
    c.bounds[pages[150], 0, 0, 3] = float("nan")
    c.table[0, 250] = c.n_pages
    c.bounds[pages[70], 0] = torch.stack([torch.full((16,), -1e30, device="cuda"), torch.full((16,), -1e30, device="cuda")]) * q[0].sum(0).sign()
    assert B.page_select(p, c.handle(p), q, 4, 0, 0).tolist() == [[[0, 1, 150, 200]]]
    chosen = B.page_select(p, c.handle(p), q, 298, 0, 0).tolist()[0][0]
    assert sorted(set(range(300)) - set(chosen)) == [70, 250]         # the lowest score, and the page that is not followed
    chosen = B.page_select(p, c.handle(p), q, 299, 0, 0).tolist()[0][0]
    assert sorted(set(range(300)) - set(chosen)) == [250]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("H", [1, 4])
def test_page_select_infinite_bounds(dtype, H):
    """Whatever the signs of the queries, a page with an infinite bound comes in before those without, through either call."""
    p = _params(H, 1, 32, dtype)
    for seed, (side, x) in enumerate([(0, -math.inf), (1, math.inf), (0, math.inf), (1, -math.inf)]):
        c = Cache([8 * 90], 1, 32, 8, dtype, seed=seed, bounds=True).fill()
        q = c.randn(1, H, 32)
        q[0, 0, 7] = 0.0
        for page, channel in ((33, 7), (61, 4), (62, 30)):
            c.bounds[int(c.table[0, page]), 0, side, channel] = x
            if x * (1 if side else -1) < 0:                       # all keys of the channel are that
                c.bounds[int(c.table[0, page]), 0, :, channel] = x
        assert B.page_select(p, c.handle(p), q, 3, 0, 0).tolist() == [[[33, 61, 62]]]
        assert B.paged_sparse_attention(p, c.handle(p), q, 3, 0, 0)[1].tolist() == [[[33, 61, 62]]]


def test_page_select_many_pages():
    """As many pages as the kernel holds, with scores that are close together."""
    n = 49152
    p = _params(4, 1, 64, BF16)
    c = Cache([n], 1, 64, 1, BF16, bounds=True, max_pages=n, fill=0.0)
    at = c.rows(0, n)
    base = c.randn(1, 1, 64)
    c.k[at] = (base + 0.01 * c.randn(n, 1, 64)).to(BF16)
    c.v[at] = c.randn(n, 1, 64)
    c.bounds[at[0], :, 0], c.bounds[at[0], :, 1] = c.k[at], c.k[at]
    q = c.randn(1, 4, 64)
    for n_sel in (1, 100, 20000, 49151):
        want = R.choose(R.scores(c, q)[0][0], n_sel, 1 if n_sel > 1 else 0, 0)
        assert B.page_select(p, c.handle(p), q, n_sel, 1 if n_sel > 1 else 0, 0).tolist() == [[want]]


def test_attention_over_a_list_of_any_order():
    """A caller's own list: any order, pages twice, entries that are no page."""
    for H, Hkv, D, dtype in [(8, 2, 128, BF16), (4, 1, 64, F32)]:
        c = Cache([100, 37, 0], Hkv, D, 8, dtype).fill()
        q = c.randn(3, H, D)
        lists = [[[12, 3, 3, 0, 7]] * Hkv, [[4, 1, 0]] * Hkv, [[]] * Hkv]
        sel = torch.tensor([[[12, 3, 3, 0, 7, -1, 99]] * Hkv, [[4, -5, 1, 0, 2 ** 31 - 1, 2, 3]] * Hkv, [[0, 1, 2, 3, 4, 5, 6]] * Hkv],
                           dtype=torch.int32, device="cuda")
        _check_attention(c, _params(H, Hkv, D, dtype), q, sel, lists)    # (of sequence 1, five pages long, five entries are read)


# ------------------------------------------------------------------------------------------ as a decoder runs them
def _decode_loop(steps, graph):
    """Compresses two layers of ragged prompts, moves what was retained into pages and decodes `steps` tokens; every step's output
    against 64 bits on the rows a plain list keeps."""
    cfg = synth.CONFIGS["ragged16"]
    lens, n_layers, page = [3000, 100, 700], 2, 32
    H, Hkv, D = cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim
    b = synth.make_batch(cfg, device="cuda", n_layers=n_layers, seq_lens=lens)
    p = B.make_params(H, Hkv, D, cfg.window, BF16, b.bitmap, cfg.vocab)
    ws = B.alloc_workspace(p, b.cu_seqlens[-1], max(lens), 3, n_layers)
    comp = B.compress_layers(p, b.q_win, b.k, b.v, b.token_ids, b.cu_seqlens, 256, cfg.candidates, ws)
    kept = comp.n_keep[0].clone()
    cs = [Cache([256 + steps] * 3, Hkv, D, page, BF16, seed=i, bounds=True) for i in range(n_layers)]
    seq_lens = kept.clone()
    freq = (500000.0 ** (-torch.arange(0, D, 2, device="cuda", dtype=torch.float64) / D)).float()
    handles = []
    for i, c in enumerate(cs):
        c.lens = seq_lens
        handles.append(c.handle(p))
        # the retained rows, packed: sequence s has kept[s] of the n_out rows
        take = torch.cat([torch.arange(n, device="cuda") + 256 * s for s, n in enumerate(kept.tolist())])
        cu = torch.tensor([0] + kept.tolist(), device="cuda").cumsum(0).to(torch.int32)
        B.paged_append(p, handles[i], comp.out_k[i].reshape(-1, Hkv, D)[take], comp.out_v[i].reshape(-1, Hkv, D)[take], cu_new=cu)
    rows = [[(comp.out_k[i, s, :n], comp.out_v[i, s, :n]) for s, n in enumerate(kept.tolist())] for i in range(n_layers)]
    # what was moved is what decoding over the compacted cache sees
    q = torch.randn(3, H, D, generator=cs[0].g, device="cuda").to(BF16)
    a = B.decode_attention(p, q, comp.out_k[0], comp.out_v[0], n_valid=kept)
    assert float((a - B.paged_attention(p, handles[0], q)).abs().max()) <= 4e-5 * float(b.v.float().abs().max())      # (rows of out_v behind n_keep hold anything)

    qkv = torch.empty(n_layers, 3, H + 2 * Hkv, D, dtype=BF16, device="cuda")
    pos = torch.tensor(lens, dtype=torch.int32, device="cuda") - 1
    outs = [torch.empty(3, H, D, device="cuda") for _ in range(2 * n_layers)]

    def step():
        seq_lens.add_(1)
        pos.add_(1)
        for i in range(n_layers):
            q, k, v = qkv[i, :, :H], qkv[i, :, H:H + Hkv], qkv[i, :, H + Hkv:]
            qr = B.paged_append(p, handles[i], k, v, q=q, positions=pos, inv_freq=freq)
            outs[2 * i].copy_(B.paged_attention(p, handles[i], qr))
            outs[2 * i + 1].copy_(B.paged_sparse_attention(p, handles[i], qr, 5)[0])

    g = None
    if graph:
        saved = seq_lens.clone(), pos.clone(), [(c.k.clone(), c.v.clone(), c.bounds.clone()) for c in cs]
        qkv.normal_()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        seq_lens.copy_(saved[0])
        pos.copy_(saved[1])
        for c, (k, v, bd) in zip(cs, saved[2]):
            c.k.copy_(k)
            c.v.copy_(v)
            c.bounds.copy_(bd)
    gen = torch.Generator(device="cuda").manual_seed(11)
    for t in range(steps):
        qkv.copy_(torch.randn(qkv.shape, generator=gen, device="cuda"))
        g.replay() if graph else step()
        at = torch.tensor(lens, device="cuda") + t
        for i, c in enumerate(cs):
            assert c.lens.tolist() == [n + t + 1 for n in kept.tolist()]
            turned = R.rotate(qkv[i, :, :H + Hkv], at, freq, False)
            for s in range(3):
                k_new = c.k[c.place(s, int(kept[s]) + t)]
                assert float((k_new.double() - turned[s, H:]).abs().max()) <= 2.0 ** -8 * float(turned[s, H:].abs().max())
                rows[i][s] = torch.cat([rows[i][s][0], k_new[None]]), torch.cat([rows[i][s][1], qkv[i, s, H + Hkv:][None]])
            q64 = turned[:, :H].to(BF16)
            got = outs[2 * i].double()
            for s in range(3):
                k, v = rows[i][s]
                for h in range(Hkv):
                    ref, _ = R.attend(q64[s, 4 * h:4 * h + 4], k[:, h], v[:, h])
                    # (a query rounded to the other neighbour moves its logits by 2^-8 of a term)
                    assert float((got[s, 4 * h:4 * h + 4] - ref).abs().max()) <= 2e-3 * float(v.float().abs().max())
            # the pages' choice, and the attention over it, from the queries that the library rotated
            if not graph:
                qr = B.paged_append(p, handles[i], qkv[i, :, H:H + Hkv], qkv[i, :, H + Hkv:], q=qkv[i, :, :H], positions=pos, inv_freq=freq)
                want = [[R.choose(x, 5, 1, 1) for x in heads] for heads in R.scores(c, qr)]
                ref, _ = R.attention(c, qr, want)
                assert float((outs[2 * i + 1].double() - ref).abs().max()) <= 2e-5 * 6
    return [o.clone() for o in outs]


def test_compress_append_and_decode():
    eager = _decode_loop(40, False)
    replayed = _decode_loop(40, True)
    for a, b in zip(eager, replayed):
        assert torch.equal(a, b)


def test_calls_on_another_stream_and_a_shared_workspace():
    p = _params(32, 8, 128, BF16)
    c = Cache([3000, 500], 8, 128, 64, BF16, bounds=True).fill()
    g = c.handle(p)
    q = c.randn(2, 32, 128)
    ref, ref_sparse = B.paged_attention(p, g, q), B.paged_sparse_attention(p, g, q, 9)
    ws = torch.empty(B.paged_workspace_bytes(p, g), dtype=torch.uint8, device="cuda").fill_(0xff)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one = B.paged_attention(p, g, q, ws=ws)
        two = B.paged_sparse_attention(p, g, q, 9, ws=ws)
        three = B.paged_attention(p, g, q, ws=ws)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(one, ref) and torch.equal(three, ref) and all(torch.equal(x, y) for x, y in zip(two, ref_sparse))


def test_refusals_on_the_gpu_leave_a_usable_context():
    p = _params(4, 2, 16, F32)
    c = Cache([5], 2, 16, 4, F32, bounds=True).fill()
    g = c.handle(p)
    x, q = c.randn(1, 2, 16), c.randn(1, 4, 16)
    for call in (lambda: B.paged_append(p, g, x, x, inv_freq=torch.zeros(9, device="cuda")), lambda: B.page_select(p, g, q, 0),
                 lambda: B.paged_sparse_attention(p, g, q, 2, 2, 1), lambda: B.paged_append(p, g, x, x, q=q, q_out=q),
                 lambda: B.paged_attention(p, g, q, ws=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(B.SablockError):
            call()
    _check_attention(c, p, q)


def test_calls_on_two_streams_at_once():
    """Nothing is shared between calls: two caches decoded on two streams at the same time, with and without scratch, say what they say alone."""
    p = _params(32, 8, 128, BF16)
    caches = [Cache([9000, 700], 8, 128, 64, BF16, seed=1, bounds=True).fill(), Cache([12000, 40, 3000], 8, 128, 32, BF16, seed=2, bounds=True).fill()]
    handles, qs = [c.handle(p) for c in caches], [c.randn(c.n_seqs, 32, 128) for c in caches]

    def both(i):
        return B.paged_attention(p, handles[i], qs[i]), *B.paged_sparse_attention(p, handles[i], qs[i], 12)
    alone = [both(i) for i in range(2)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(both(i))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for one in got[i] for a, b in zip(one, alone[i]))


def test_a_cache_on_another_device_than_the_current_one_is_refused():
    p = _params(4, 2, 16, F32)
    c = Cache([5], 2, 16, 4, F32, bounds=True).fill()
    g = c.handle(p)
    g._index += 1                                             # as if it were on the next GPU
    x, q = c.randn(1, 2, 16), c.randn(1, 4, 16)
    for call in (lambda: B.paged_append(p, g, x, x), lambda: B.paged_attention(p, g, q), lambda: B.page_select(p, g, q, 2),
                 lambda: B.paged_sparse_attention(p, g, q, 2)):
        with pytest.raises(ValueError):
            call()


def test_another_parameter_block_than_the_caches():
    p = _params(4, 2, 16, F32)
    c = Cache([5], 2, 16, 4, F32, bounds=True).fill()
    g = c.handle(p)
    x, q = c.randn(1, 2, 16), c.randn(1, 4, 16)
    same, others = _params(4, 2, 16, F32), [_params(8, 2, 16, F32), _params(4, 4, 16, F32), _params(4, 2, 32, F32), _params(4, 2, 16, BF16)]
    assert torch.equal(B.paged_attention(p, g, q), B.paged_attention(same, g, q))
    for o in others:
        for call in (lambda: B.paged_append(o, g, x, x), lambda: B.paged_attention(o, g, q), lambda: B.page_select(o, g, q, 2),
                     lambda: B.paged_sparse_attention(o, g, q, 2)):
            with pytest.raises((ValueError, TypeError)):
                call()


def test_as_many_sequences_as_a_call_takes():
    n = 4096
    p = _params(2, 1, 64, BF16)
    lens = [(i * 5) % 23 for i in range(n)]
    c = Cache(lens, 1, 64, 8, BF16, fill=0.0, bounds=True)
    new = [min(x, i % 4) for i, x in enumerate(lens)]
    for s, x in enumerate(lens):
        at = c.rows(s, x - new[s])
        c.k[at], c.v[at] = c.randn(x - new[s], 1, 64), c.randn(x - new[s], 1, 64)
        c.set_bounds(s, x - new[s])
    k, v = c.randn(sum(new), 1, 64), c.randn(sum(new), 1, 64)
    g = c.handle(p)
    B.paged_append(p, g, k, v, cu_new=torch.tensor([0] + new, device="cuda").cumsum(0).to(torch.int32))
    kept, t = c.bounds.clone(), 0
    for s, x in enumerate(lens):
        for r in range(x - new[s], x):
            assert torch.equal(c.k[c.place(s, r)], k[t]) and torch.equal(c.v[c.place(s, r)], v[t])
            t += 1
        if new[s]:
            c.set_bounds(s, x)
    assert torch.equal(kept, c.bounds)
    q = c.randn(n, 2, 64)
    _check_attention(c, p, q)
    want = [[R.choose(x, 2, 0, 1) for x in heads] for heads in R.scores(c, q)]
    sel = B.page_select(p, g, q, 2, 0, 1)
    assert sel.tolist() == [[x + [-1] * (2 - len(x)) for x in heads] for heads in want]
    _check_attention(c, p, q, sel, want)


def test_one_page_per_sequence():
    """A cache of long rows that are not split at all: the page is the sequence."""
    p = _params(4, 2, 64, BF16)
    c = Cache([0, 0], 2, 64, 3000, BF16, bounds=True, max_pages=1, spare=0)
    g = c.handle(p)
    new = [2500, 130]
    for part in (0.5, 1.0):                                  # in two parts: the second widens the bounds of the first
        had = c.lens.tolist()
        c.lens.copy_(torch.tensor([int(x * part) for x in new]))
        n = [a - b for a, b in zip(c.lens.tolist(), had)]
        k, v = c.randn(sum(n), 2, 64), c.randn(sum(n), 2, 64)
        B.paged_append(p, g, k, v, cu_new=torch.tensor([0] + n, device="cuda").cumsum(0).to(torch.int32))
        t = 0
        for s in range(2):
            page = int(c.table[s, 0])
            assert torch.equal(c.k[page, had[s]:had[s] + n[s]], k[t:t + n[s]]) and torch.equal(c.v[page, had[s]:had[s] + n[s]], v[t:t + n[s]])
            t += n[s]
        got = c.bounds.clone()
        for s in range(2):
            c.set_bounds(s, c.lens.tolist()[s])
        assert torch.equal(got, c.bounds)
    q = c.randn(2, 4, 64)
    _check_attention(c, p, q)
    assert B.page_select(p, g, q, 3).tolist() == [[[0, -1, -1]] * 2] * 2


def test_append_through_ctypes_and_through_the_module():
    """The binding without its marshalling module, and a caller's own buffer for the queries, do the same."""
    p = _params(8, 2, 64, BF16)
    outs = []
    for slow, own in ((False, False), (True, False), (False, True)):
        c = Cache([40, 9], 2, 64, 16, BF16, seed=4, bounds=True, fill=0.0)
        g = c.handle(p)
        if slow:
            g._fast = None
        qkv = c.randn(7, 12, 64)
        buf = torch.empty(7, 8, 64, dtype=BF16, device="cuda") if own else None
        freq = torch.linspace(1.0, 0.001, 32, device="cuda")
        q = B.paged_append(p, g, qkv[:, 8:10], qkv[:, 10:], q=qkv[:, :8], inv_freq=freq, cu_new=torch.tensor([0, 4, 7], dtype=torch.int32, device="cuda"),
                           positions=torch.arange(7, dtype=torch.int32, device="cuda") * 9, q_out=buf)
        assert q.is_contiguous()
        outs.append((q, c.k, c.v, c.bounds))
    for other in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(outs[0], other))
    with pytest.raises(ValueError):
        B.paged_append(p, g, qkv[:, 8:10], qkv[:, 9:10])
    with pytest.raises(TypeError):
        B.paged_append(p, g, qkv[:, 8:10].float(), qkv[:, 10:])


def test_a_graph_whose_sequences_grow_over_the_rows_of_one_launch():
    """A captured attention replayed with other lengths, from none to the table's, on either side of every rule that the host cannot see."""
    for max_pages, page in ((20, 16), (300, 64)):                 # one launch; shares
        p = _params(8, 2, 128, BF16)
        full = max_pages * page
        c = Cache([full] * 3, 2, 128, page, BF16, seed=max_pages, bounds=True, max_pages=max_pages).fill()
        g = c.handle(p)
        q = c.randn(3, 8, 128)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            B.paged_attention(p, g, q, want_lse=True)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out, lse = B.paged_attention(p, g, q, want_lse=True)
            sparse, sel = B.paged_sparse_attention(p, g, q, 6)
        for lens in ([0, 0, 0], [1, 0, full], [full - 1, 17, page * 6], [page * 6 + 1, 5, 64]):
            c.lens.copy_(torch.tensor(lens))
            for pages in range(3):
                c.set_bounds(pages, lens[pages])
            graph.replay()
            ref, ref_lse = R.attention(c, q)
            assert float((out.double() - ref).abs().max()) <= 2e-5 * 6
            want = [[R.choose(x, 6, 1, 1) for x in heads] for heads in R.scores(c, q)]
            assert sel.tolist() == [[x + [-1] * (6 - len(x)) for x in heads] for heads in want]
            assert float((sparse.double() - R.attention(c, q, want)[0]).abs().max()) <= 2e-5 * 6
