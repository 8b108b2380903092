"""What the binding's calls over a paged cache do with a call that they refuse, with blocks and tensors that change, with nothing to do:
on the host (no GPU), the entry points themselves replaced where a good call would enqueue work."""
import ctypes as C
import random

import pytest
import torch

from paper_2510_22556_b200 import binding as B
from paper_2510_22556_b200 import build as build_lib
from paper_2510_22556_b200.build import build_test_hooks


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_lib()
    B.lib()


def _params(H=8, Hkv=4, D=16, dtype=torch.float32):
    return B.make_params(H, Hkv, D, 1, dtype)


def _cache(p, seqs=2, page=4, max_pages=3, n_pages=8):
    """Handle of a small cache on the CPU."""
    dt, hkv, d = {B.F32: torch.float32, B.BF16: torch.bfloat16}[p.dtype], p.n_kv_heads, p.head_dim
    k, v = (torch.zeros(n_pages, page, hkv, d, dtype=dt) for _ in range(2))
    return B.make_pages(p, k, v, torch.zeros(seqs, max_pages, dtype=torch.int32), torch.zeros(seqs, dtype=torch.int32), torch.zeros(n_pages, hkv, 2, d, dtype=dt))


def _like(p, g, n):
    """What a call allocates: bytes of scratch, shape of the page list."""
    ws, sel = B._like(p, g, n)
    return None if ws is None else ws.numel(), tuple(sel.shape)


@pytest.mark.parametrize("why", ["heads", "kv_heads", "head_dim", "device"])
def test_a_refused_call_leaves_the_handle_as_it_was(monkeypatch, why):
    """The scratch and the page list of the next good call have the sizes that they have on a handle that no call was refused on."""
    p = _params()
    g, fresh, q = _cache(p), _cache(p), torch.zeros(2, 8, 16)
    bad = {"heads": _params(H=32), "kv_heads": _params(Hkv=2), "head_dim": _params(D=4), "device": p}[why]
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 3, raising=False)
    for call in (lambda: B.paged_attention(bad, g, q), lambda: B.paged_attention(bad, g, q, selected=torch.zeros(2, bad.n_kv_heads, 2, dtype=torch.int32)),
                 lambda: B.page_select(bad, g, q, 2), lambda: B.paged_sparse_attention(bad, g, q, 2)):
        with pytest.raises(ValueError):
            call()
    assert not g._like
    for n in (0, -1, 2):
        assert _like(p, g, n) == _like(p, fresh, n)


@pytest.mark.parametrize("field,value", [("n_q_heads", 16), ("n_kv_heads", 2), ("head_dim", 32), ("dtype", B.BF16)])
def test_a_block_whose_sizes_changed_after_the_cache_was_described(field, value):
    """The block is the caller's to change; with other sizes than the cache's it is refused though it is the same block."""
    p = _params()
    g = _cache(p)
    setattr(p, field, value)
    q, x, sel = torch.zeros(2, 8, 16), torch.zeros(2, p.n_kv_heads, p.head_dim), torch.zeros(2, p.n_kv_heads, 2, dtype=torch.int32)
    for call in (lambda: B.paged_append(p, g, x, x), lambda: B.paged_attention(p, g, q), lambda: B.paged_attention(p, g, q, selected=sel),
                 lambda: B.page_select(p, g, q, 2), lambda: B.paged_sparse_attention(p, g, q, 2)):
        with pytest.raises(ValueError, match="other sizes"):
            call()
    assert not g._like


class _Entry:
    """Stands in for the library: notes the arguments of the entry points that enqueue work, and enqueues nothing."""

    def __init__(self, real):
        self.real, self.calls = real, []

    def __getattr__(self, name):
        if name in ("paged_append", "paged_attention", "page_select", "paged_sparse_attention"):
            return lambda *a: self.calls.append((name, a)) or 0
        return getattr(self.real, name)


@pytest.fixture
def entry(monkeypatch):
    """Good calls on CPU tensors go through the binding and end there."""
    e = _Entry(B.lib())
    monkeypatch.setattr(B, "lib", lambda: e)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0, raising=False)
    return e


def test_scratch_that_is_not_what_its_size_says_is_refused(entry):
    """Scratch on another device, or one element expanded, has an address and a number of elements that the entry points would believe."""
    p = _params()
    g, q = _cache(p), torch.zeros(2, 8, 16)
    n = B.paged_workspace_bytes(p, g)
    calls = (lambda ws: B.paged_attention(p, g, q, ws=ws), lambda ws: B.paged_sparse_attention(p, g, q, 2, ws=ws))
    for ws in (torch.zeros(1, dtype=torch.uint8).expand(n), torch.zeros(2 * n, dtype=torch.uint8)[::2], torch.empty(n, dtype=torch.uint8, device="meta"), bytearray(n)):
        for call in calls:
            with pytest.raises((TypeError, ValueError)):
                call(ws)
    assert not entry.calls
    ws = torch.zeros(n, dtype=torch.uint8)
    for call in calls:
        call(ws)
    assert [a[-3:] for _, a in entry.calls] == [(ws.data_ptr(), n, 0)] * 2


def test_an_empty_list_of_pages_is_not_all_of_them(entry):
    """A list without entries has no address, which to the entry point says all rows."""
    p = _params()
    g, q = _cache(p), torch.zeros(2, 8, 16)
    for sel in (torch.zeros(2, 4, 0, dtype=torch.int32), torch.zeros(2, 4, 3, dtype=torch.int32)[..., :0]):
        with pytest.raises(B.SablockError) as e:
            B.paged_attention(p, g, q, selected=sel)
        assert e.value.code == 1
    assert not entry.calls
    sel = torch.zeros(2, 4, 1, dtype=torch.int32)
    B.paged_attention(p, g, q, selected=sel)
    assert entry.calls[0][1][3:5] == (sel.data_ptr(), 1)


@pytest.fixture
def module(monkeypatch, entry):
    """Appending goes through the marshalling module, CPU tensors too: the arguments of the entry point that it would call."""
    fast = pytest.importorskip("paper_2510_22556_b200._fastcall")
    got = []
    fn = C.CFUNCTYPE(C.c_int, *[C.c_uint64] * 16)(lambda *a: got.append(a) or 0)
    entry.append_step = fast.bind_append(C.cast(fn, C.c_void_p).value)
    entry.keep = fn
    return got


def _module_handle(p, **kw):
    g = _cache(p, **kw)
    g._fast = g._dtype, g._device, g.n_seqs, p.n_kv_heads, p.n_q_heads, p.head_dim, torch.int32, torch.float32, torch.empty_like
    return g


@pytest.mark.parametrize("through_module", [False, True])
@pytest.mark.parametrize("strides", [(8, 16, 1), (16, 16, 1), (48, 16, 1), (64, 16, 1), (120, 16, 1)])
def test_the_rotated_queries_lie_side_by_side_whatever_the_queries_strides(module, entry, through_module, strides):
    """Tokens that overlap (a stride below a token's heads) may be read, but what comes back is written token after token."""
    p = _params(H=4, Hkv=1)
    g = _module_handle(p, seqs=5) if through_module else _cache(p, seqs=5)
    q, x = torch.zeros(1000).as_strided((5, 4, 16), strides), torch.zeros(5, 1, 16)
    out = B.paged_append(p, g, x, x, q=q)
    assert out.shape == q.shape and out.is_contiguous()
    at = module[0] if module else entry.calls[0][1]
    assert at[8:11] == (q.data_ptr(), strides[0], out.data_ptr())
    assert len(module) + len(entry.calls) == 1 and bool(module) == (through_module and strides[0] >= 64)


class _Named(torch.Tensor):
    """A caller's own kind of tensor: what is made like it is of that kind too."""


def test_an_append_of_another_kind_of_tensor_is_enqueued_once(module, entry):
    p = _params(H=4, Hkv=1)
    g, x, q = _module_handle(p, seqs=5), torch.zeros(5, 1, 16), torch.zeros(5, 4, 16).as_subclass(_Named)
    out = B.paged_append(p, g, x, x, q=q)
    assert len(module) == 1 and not entry.calls
    assert out.shape == q.shape and out.data_ptr() == module[0][10]


def test_a_status_of_the_module_is_raised_once(module, entry, monkeypatch):
    p = _params(H=4, Hkv=1)
    g, x = _module_handle(p, seqs=5), torch.zeros(5, 1, 16)
    entry.append_step = lambda *a: module.append(a) or 4
    with pytest.raises(B.SablockError) as e:
        B.paged_append(p, g, x, x)
    assert e.value.code == 4 and len(module) == 1 and not entry.calls


@pytest.mark.parametrize("through_module", [False, True])
def test_appending_no_tokens(monkeypatch, through_module):
    """A step in which no sequence has new tokens: tensors without elements have no address, and nothing is wrong with that."""
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0, raising=False)
    p = _params(H=4, Hkv=1)
    g = _module_handle(p) if through_module else _cache(p)
    x, q, cu = torch.zeros(0, 1, 16), torch.zeros(0, 4, 16), torch.zeros(3, dtype=torch.int32)
    pos, freq = torch.zeros(0, dtype=torch.int32), torch.ones(8)
    assert B.paged_append(p, g, x, x, cu_new=cu) is None
    out = B.paged_append(p, g, x, x, q=q, positions=pos, inv_freq=freq, cu_new=cu)
    assert out.shape == (0, 4, 16) and B.last_launch_count() == 0
    with pytest.raises(B.SablockError):            # one token each is not none
        B.paged_append(p, g, x, x)
    with pytest.raises(B.SablockError):
        B.paged_append(p, g, x, x, cu_new=cu, inv_freq=torch.ones(9))


FAKE = 1 << 30                                     # never dereferenced


@pytest.mark.parametrize("array", ["q", "k", "v"])
@pytest.mark.parametrize("stride", [0, 768])       # contiguous; the parts of one projection's output
def test_rotated_queries_over_an_array_that_is_read(array, stride):
    """Another CTA may not have read the tokens that such a write falls on."""
    p, n, heads = _params(8, 2, 64, torch.bfloat16), 5, 8 if array == "q" else 2
    g = B.Pages()
    g.k, g.v, g.table, g.seq_lens = FAKE << 1, FAKE << 2, FAKE << 3, FAKE << 4
    g.n_seqs, g.n_pages, g.page_size, g.max_pages = n, 100, 64, 20
    at = dict(q=FAKE + (1 << 20), k=FAKE + (2 << 20), v=FAKE + (3 << 20))
    last = at[array] + ((n - 1) * (stride or heads * 64) + heads * 64) * 2         # behind the last token
    for q_out in (at[array], last - 16, at[array] - n * 8 * 64 * 2 + 16):
        code = B.lib().paged_append(C.addressof(p), C.addressof(g), n, None, at["k"], stride, at["v"], stride, at["q"], stride, q_out, None, None, 0, 0, None)
        assert code == 1


def test_what_meets_the_rows_of_an_array():
    """Bytes against rows that lie apart, side by side or over one another, byte by byte."""
    hooks = C.CDLL(build_test_hooks())
    hooks.sablock_test_meets_rows.argtypes = [C.c_size_t] * 6
    r = random.Random(3)
    seen = [0, 0]
    for _ in range(4000):
        out, n_out, at, row, step, n = r.randint(50, 150), r.randint(1, 40), r.randint(50, 150), r.randint(1, 20), r.randint(1, 40), r.randint(1, 6)
        rows = {at + i * step + b for i in range(n) for b in range(row)}
        want = not rows.isdisjoint(range(out, out + n_out))
        seen[want] += 1
        assert bool(hooks.sablock_test_meets_rows(out, n_out, at, row, step, n)) == want
    assert min(seen) > 800


@pytest.mark.parametrize("n,kw,code", [
    (0, {}, 1), (-1, {}, 1), (-5, {}, 1), (4, dict(n_first=-1), 1), (4, dict(n_first=3, n_last=2), 1), (4, dict(n_first=1 << 32), 1), (4, dict(n_last=(1 << 32) + 1), 1),
    (1 << 29, {}, 2), ((1 << 32) + 4, {}, 2), (1 << 45, {}, 2)])
def test_a_choice_that_cannot_be_is_refused_before_its_list_is_allocated(entry, n, kw, code):
    """Pages of four rows: 2^28 pages are as many rows as a sequence can have.  Numbers past 32 bits are not cut to their low ones."""
    p = _params()
    g, q = _cache(p), torch.zeros(2, 8, 16)
    for call in (lambda: B.page_select(p, g, q, n, **kw), lambda: B.paged_sparse_attention(p, g, q, n, **kw)):
        with pytest.raises(B.SablockError) as e:
            call()
        assert e.value.code == code
    assert not entry.calls and not g._like


def test_scratch_of_a_choice_that_cannot_be():
    p = _params()
    g = _cache(p)
    need = [int(B.lib().sablock_paged_workspace_bytes(C.addressof(p), C.addressof(g), n)) for n in (-1, 0, 1 << 28, (1 << 28) + 1, -2)]
    assert min(need[:3]) > 0 and need[3:] == [0, 0]
