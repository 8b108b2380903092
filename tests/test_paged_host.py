"""The paged cache's calls on the host (no GPU): arguments that are refused before anything is enqueued, what the binding makes
of tensors, and the host arithmetic that the kernels share."""
import ctypes as C
import random

import pytest
import torch

from paper_2510_22556_b200 import binding as B
from paper_2510_22556_b200 import build as build_lib
from paper_2510_22556_b200.build import build_test_hooks

INVALID, UNSUPPORTED, TOO_SMALL = 1, 2, 3
FAKE = 1 << 20                                     # never dereferenced


@pytest.fixture(scope="module")
def lib():
    build_lib()
    return B.lib()


@pytest.fixture(scope="module")
def hooks():
    l = C.CDLL(build_test_hooks())
    l.sablock_test_append_runs.restype = C.c_longlong
    l.sablock_test_append_runs.argtypes = [C.c_longlong, C.c_int, C.c_int, C.c_int]
    return l


def _params(**kw):
    base = dict(n_q_heads=32, n_kv_heads=8, head_dim=128, window=32, dtype=torch.bfloat16)
    base.update(kw)
    return B.make_params(**base)


def _pages(**kw):
    g = B.Pages()
    for name in ("k", "v", "bounds", "table", "seq_lens"):
        setattr(g, name, FAKE)
    g.n_seqs, g.n_pages, g.page_size, g.max_pages = 3, 100, 64, 20
    for k, v in kw.items():
        setattr(g, k, v)
    return g


NAMES = ("append", "attend", "select", "sparse")


def _call(l, name, p, g, **kw):
    """Status of an entry point on arguments of which something is wrong (good ones would enqueue work)."""
    P, G = C.addressof(p) if p is not None else None, C.addressof(g) if g is not None else None
    a = dict(n=3, cu=None, k=FAKE, ks=0, v=FAKE, vs=0, q=FAKE, qs=0, q_out=FAKE * 64, inv=FAKE, rd=128, sel=FAKE, n_sel=4, first=1, last=1,
             out=FAKE, ws=FAKE, ws_bytes=1 << 40)
    a.update(kw)
    if name == "append":
        return l.paged_append(P, G, a["n"], a["cu"], a["k"], a["ks"], a["v"], a["vs"], a["q"], a["qs"], a["q_out"], None, a["inv"], a["rd"], 0, None)
    if name == "attend":
        return l.paged_attention(P, G, a["q"], a["sel"], a["n_sel"], a["out"], None, a["ws"], a["ws_bytes"], None)
    if name == "select":
        return l.page_select(P, G, a["q"], a["n_sel"], a["first"], a["last"], a["sel"], None)
    return l.paged_sparse_attention(P, G, a["q"], a["n_sel"], a["first"], a["last"], a["sel"], a["out"], None, a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("params,pages,code", [
    (dict(n_q_heads=30), {}, INVALID), (dict(head_dim=0), {}, INVALID), (dict(head_dim=100), {}, UNSUPPORTED), (dict(head_dim=264), {}, UNSUPPORTED),
    (dict(n_q_heads=8192, n_kv_heads=1), {}, UNSUPPORTED), ({}, dict(k=None), INVALID), ({}, dict(v=None), INVALID), ({}, dict(table=None), INVALID),
    ({}, dict(seq_lens=None), INVALID), ({}, dict(n_seqs=0), INVALID), ({}, dict(n_pages=0), INVALID), ({}, dict(page_size=0), INVALID),
    ({}, dict(max_pages=-1), INVALID), ({}, dict(n_seqs=4097), UNSUPPORTED), ({}, dict(max_pages=1 << 25), UNSUPPORTED),
    ({}, dict(k_stride_row=-8), INVALID), ({}, dict(v_stride_page=4), UNSUPPORTED), ({}, dict(k_stride_head=129), UNSUPPORTED),
    ({}, dict(table_stride=19), INVALID), ({}, dict(k=FAKE + 8), UNSUPPORTED), ({}, dict(bounds=FAKE + 2), UNSUPPORTED),
])
def test_caches_that_every_call_refuses(lib, params, pages, code):
    p, g = _params(**params), _pages(**pages)
    assert [_call(lib, name, p, g) for name in NAMES] == [code] * 4
    assert lib.sablock_paged_workspace_bytes(C.addressof(p), C.addressof(g), -1) == 0


def test_null_blocks(lib):
    for name in NAMES:
        assert _call(lib, name, None, _pages()) == INVALID == _call(lib, name, _params(), None)


@pytest.mark.parametrize("kw,who,code", [
    (dict(k=None), ["append"], INVALID), (dict(v=None), ["append"], INVALID), (dict(n=-1), ["append"], INVALID), (dict(n=4), ["append"], INVALID),
    (dict(q_out=None), ["append"], INVALID), (dict(q_out=FAKE), ["append"], INVALID), (dict(q_out=FAKE + 2 * 4096 * 3 - 16), ["append"], INVALID),
    (dict(qs=-1), ["append"], INVALID), (dict(ks=1025), ["append"], UNSUPPORTED), (dict(v=FAKE + 2), ["append"], UNSUPPORTED),
    (dict(rd=0), ["append"], INVALID), (dict(rd=130), ["append"], INVALID), (dict(rd=7), ["append"], INVALID), (dict(inv=None), ["append"], INVALID),
    (dict(q=None), ["attend", "select", "sparse", "append"], INVALID), (dict(q=FAKE + 4), ["attend", "select", "sparse", "append"], UNSUPPORTED),
    (dict(out=None), ["attend", "sparse"], INVALID), (dict(n_sel=0), ["attend", "select", "sparse"], INVALID),
    (dict(sel=None), ["attend", "select", "sparse"], INVALID), (dict(first=-1), ["select", "sparse"], INVALID),
    (dict(first=3, last=2), ["select", "sparse"], INVALID), (dict(last=1 << 30), ["select", "sparse"], INVALID),
    (dict(n_sel=1 << 30), ["attend", "select", "sparse"], UNSUPPORTED),
    (dict(ws=None), ["attend"], TOO_SMALL), (dict(ws_bytes=64), ["attend"], TOO_SMALL), (dict(ws=FAKE + 8), ["attend"], INVALID),
])
def test_arguments_that_are_refused(lib, kw, who, code):
    for name in who:
        assert _call(lib, name, _params(), _pages(), **kw) == code


def test_selection_needs_bounds_and_a_table_that_fits(lib):
    p = _params()
    P = C.addressof(p)
    for g, code in ((_pages(bounds=None), INVALID), (_pages(max_pages=49153, page_size=16), UNSUPPORTED)):
        assert lib.page_select(P, C.addressof(g), FAKE, 4, 1, 1, FAKE, None) == code
        assert lib.paged_sparse_attention(P, C.addressof(g), FAKE, 4, 1, 1, FAKE, FAKE, None, FAKE, 1 << 40, None) == code


def test_scratch(lib):
    """Short rows and chosen pages go out in one launch without scratch; long ones, fp32, a list that is given need it."""
    p = _params()
    short, long_, f32 = _pages(), _pages(max_pages=2000, page_size=64), _params(dtype=torch.float32)
    need = lambda q, g, n: int(lib.sablock_paged_workspace_bytes(C.addressof(q), C.addressof(g), n))  # noqa: E731
    full = need(p, short, -1)
    assert full > 1 << 20 and need(p, short, 0) == 16 and need(p, long_, 0) == full == need(p, long_, -1)
    assert need(p, _pages(n_seqs=16, max_pages=500, page_size=32), 48) == 16 and need(p, _pages(n_seqs=1, max_pages=2049), 64) == full
    assert need(p, short, 2000) == full and need(f32, short, 0) > 16 and need(f32, short, 4) > 16
    for g, kw, code in ((long_, dict(ws=None), TOO_SMALL), (long_, dict(ws_bytes=full - 1), TOO_SMALL), (long_, dict(ws=FAKE + 8), INVALID)):
        assert _call(lib, "attend", p, g, sel=None, n_sel=0, **kw) == code == _call(lib, "sparse", p, _pages(n_seqs=1, max_pages=2049), n_sel=64, **kw)
    assert B.last_launch_count() == 0


def test_appending_nothing_is_no_error(lib):
    p, g = _params(), _pages()
    assert lib.paged_append(C.addressof(p), C.addressof(g), 0, FAKE, FAKE, 0, FAKE, 0, None, 0, None, None, None, 0, 0, None) == 0
    assert B.last_launch_count() == 0


# ------------------------------------------------------------------------------------------ the binding
def _tensors(n_pages=6, ps=4, hkv=2, d=16, seqs=2, max_pages=3, dtype=torch.float32):
    return (torch.zeros(n_pages, ps, hkv, d, dtype=dtype), torch.zeros(n_pages, ps, hkv, d, dtype=dtype),
            torch.zeros(seqs, max_pages, dtype=torch.int32), torch.zeros(seqs, dtype=torch.int32))


def test_make_pages_reads_strides_off_the_tensors(lib):
    p = _params(n_q_heads=4, n_kv_heads=2, head_dim=16, dtype=torch.float32)
    kv = torch.zeros(6, 2, 2, 4, 16)                       # page, K or V, head, slot, channel
    k, v = kv[:, 0].transpose(1, 2), kv[:, 1].transpose(1, 2)
    table = torch.zeros(2, 5, dtype=torch.int32)[:, 1:4]
    g = B.make_pages(p, k, v, table, torch.zeros(2, dtype=torch.int32), torch.zeros(6, 2, 2, 16))
    assert (g.k, g.v, g.table) == (k.data_ptr(), v.data_ptr(), table.data_ptr())
    assert (g.k_stride_page, g.k_stride_row, g.k_stride_head) == (256, 16, 64) == (g.v_stride_page, g.v_stride_row, g.v_stride_head)
    assert (g.n_seqs, g.n_pages, g.page_size, g.max_pages, g.table_stride) == (2, 6, 4, 3, 5)
    assert B.paged_workspace_bytes(p, g) > 16


def test_make_pages_refuses(lib):
    p = _params(n_q_heads=4, n_kv_heads=2, head_dim=16, dtype=torch.float32)
    k, v, table, lens = _tensors()
    for bad in [(k.bfloat16(), v, table, lens), (k, v[:5], table, lens), (k, v, table.long(), lens), (k, v, table, lens[:1]), (k[0], v[0], table, lens),
                (k.flip(3).transpose(2, 3).contiguous().transpose(2, 3), v, table, lens), (k, v, table.t().contiguous().t(), lens),
                (k[:1].expand(6, -1, -1, -1), v, table, lens), (k, v[:, :, :1].expand(-1, -1, 2, -1), table, lens), (k, v[:, :1].expand(-1, 4, -1, -1), table, lens),
                (k, v, table[:1].expand(2, -1), lens), (k, v, torch.zeros(9, dtype=torch.int32).as_strided((2, 3), (1, 1)), lens),
                (k, v, table, lens, torch.zeros(6, 2, 16)), (k, v, table, lens, torch.zeros(6, 2, 2, 32)[..., ::2])]:
        with pytest.raises((TypeError, ValueError)):
            B.make_pages(p, *bad)


def test_calls_refuse_tensors_that_do_not_fit(lib):
    p = _params(n_q_heads=4, n_kv_heads=2, head_dim=16, dtype=torch.float32)
    g = B.make_pages(p, *_tensors(), torch.zeros(6, 2, 2, 16))
    x, q = torch.zeros(2, 2, 16), torch.zeros(2, 4, 16)
    pos, freq = torch.zeros(2, dtype=torch.int32), torch.zeros(8)
    for a, kw in [((x[:1], x), {}), ((x.half(), x), {}), ((x, x), dict(q=q[:, :3])), ((x, x), dict(q=q.transpose(1, 2).contiguous().transpose(1, 2))),
                  ((x, x), dict(q_out=q)), ((x, x), dict(q=q, q_out=q[:1])), ((x, x), dict(positions=pos.long())), ((x, x), dict(positions=pos[:1])),
                  ((x[:1].expand(2, -1, -1), x), {}), ((x, x), dict(q=q[:1].expand(2, -1, -1))), ((x, x), dict(inv_freq=freq.double())), ((x, x), dict(cu_new=pos)), ((x, x), dict(inv_freq=torch.zeros(16)[::2]))]:
        with pytest.raises((TypeError, ValueError)):
            B.paged_append(p, g, *a, **kw)
    for fn in (lambda t: B.paged_attention(p, g, t), lambda t: B.page_select(p, g, t, 2), lambda t: B.paged_sparse_attention(p, g, t, 2)):
        for t in (q[:1], q.double(), q[..., :8], torch.zeros(4, 2, 16).transpose(0, 1)):
            with pytest.raises((TypeError, ValueError)):
                fn(t)
    for sel in (torch.zeros(2, 2, 3), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 4, 3, dtype=torch.int32)):
        with pytest.raises((TypeError, ValueError)):
            B.paged_attention(p, g, q, selected=sel)


@pytest.mark.parametrize("n,heads,d", [(3, 2, 16), (1, 2, 16), (0, 2, 16), (3, 1, 16), (3, 2, 1)])
def test_tensor_checks_of_the_marshalling_module(n, heads, d):
    """The C checks say what the Python ones say."""
    fast = pytest.importorskip("paper_2510_22556_b200._fastcall")
    cpu, wide = torch.device("cpu"), torch.zeros(max(n, 1) * 2, heads + 3, d)
    views = [torch.zeros(n, heads, d), wide[:n, 1:1 + heads], wide[::2][:n, :heads], torch.zeros(n, d, heads).transpose(1, 2), torch.zeros(n, heads, d, dtype=torch.int32),
             torch.zeros(n + 1, heads, d), torch.zeros(n, heads * d), torch.zeros(1, heads, d).expand(n, heads, d), torch.zeros(n, heads, d, device="meta"),
             torch.zeros(n, 1, d).expand(n, heads, d)]
    got = []
    for t in views:
        slow = -1
        if t.dtype == torch.float32 and t.device == cpu and t.shape == (n, heads, d) and \
                not (n and ((d > 1 and t.stride(2) != 1) or (heads > 1 and t.stride(1) != d) or (n > 1 and t.stride(0) == 0))):
            slow = t.stride(0) if n > 1 else 0
        got.append(fast.token_stride(t, torch.float32, cpu, n, heads, d))
        assert got[-1] == slow
        assert fast.fits(t, torch.float32, cpu, (n, heads, d)) is (t.dtype == torch.float32 and t.device == cpu and t.shape == (n, heads, d) and
                                                                   t.is_contiguous())
    if n == 3 and heads == 2 and d == 16:
        assert got[:3] == [32, 5 * 16, 10 * 16] and got[4] == -1
    for bad in [(), (views[0],), (views[0], torch.float32, cpu, n, heads)]:
        with pytest.raises(TypeError):
            fast.fits(*bad)
        with pytest.raises(TypeError):
            fast.token_stride(*bad)
    with pytest.raises(AttributeError):
        fast.fits(5, torch.float32, cpu, (n, heads, d))


# ------------------------------------------------------------------------------------------ host arithmetic
@pytest.mark.parametrize("d", [1, 2, 3, 5, 7, 16, 20, 64, 100, 127, 128, 641, 65535, 65536, (1 << 20) + 7, (1 << 30) - 1, 1 << 30])
def test_fast_division(hooks, d):
    r = random.Random(d)
    top = (1 << 31) - 1
    near = [q * d + e for q in (0, 1, 2, top // d - 1, top // d) for e in (-1, 0, 1)]
    for n in near + [top, top - 1] + [r.randrange(top) for _ in range(2000)]:
        if 0 <= n <= top:
            assert hooks.sablock_test_fast_div(n, d) == n // d


def test_runs_of_an_append_fit_the_grid(hooks):
    """Every sequence's rows [L - n, L) cut at multiples of the run length: never more runs than the grid has CTAs."""
    r = random.Random(5)
    for _ in range(3000):
        n_seqs, run = r.randint(1, 9), r.choice([1, 2, 3, 8, 16, 64])
        new = [r.choice([0, 1, 2, r.randint(0, 200)]) for _ in range(n_seqs)]
        runs = 0
        for n in new:
            end = n + r.randint(0, 300)
            runs += (end - 1) // run - (end - n) // run + 1 if n else 0
        assert runs <= hooks.sablock_test_append_runs(sum(new), n_seqs, run, 0)
    assert hooks.sablock_test_append_runs(7, 7, 64, 1) == 7
