"""Calls over a paged cache on the GPU after calls that were refused, and with tensors of unusual layouts."""
import pytest
import torch

import paged_reference as R
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


def test_good_calls_after_refused_ones():
    """A handle that calls with other parameter blocks were refused on does what one does that they were not."""
    p = _params(8, 4, 64, F32)
    c = Cache([3000, 500], 4, 64, 16, F32, bounds=True).fill()
    g, fresh, q = c.handle(p), c.handle(p), c.randn(2, 8, 64)
    for o in (_params(8, 2, 64, F32), _params(8, 4, 4, F32), _params(32, 4, 64, F32)):
        for call in (lambda: B.paged_attention(o, g, q), lambda: B.page_select(o, g, q, 6), lambda: B.paged_sparse_attention(o, g, q, 6)):
            with pytest.raises(ValueError):
                call()
    want = [[R.choose(x, 6, 1, 1) for x in heads] for heads in R.scores(c, q)]
    assert B.page_select(p, g, q, 6).tolist() == want
    assert torch.equal(B.paged_attention(p, g, q), B.paged_attention(p, fresh, q))
    assert all(torch.equal(a, b) for a, b in zip(B.paged_sparse_attention(p, g, q, 6), B.paged_sparse_attention(p, fresh, q, 6)))


@pytest.mark.parametrize("stride", [16, 64, 128, 512, 1000])
def test_append_with_queries_that_overlap(stride):
    """Query tokens that lie closer than their heads are many (a window that slides) are read as they lie and come back token after token."""
    p, n = _params(8, 2, 64, F32), 7
    c = Cache([4, 3], 2, 64, 16, F32, fill=0.0)
    q = c.randn(n * 1000 + 512).as_strided((n, 8, 64), (stride, 64, 1))
    x, pos = c.randn(n, 2, 64), torch.arange(n, dtype=torch.int32, device="cuda") * 11
    freq, cu = torch.linspace(1.0, 0.001, 32, device="cuda"), torch.tensor([0, 4, 7], dtype=torch.int32, device="cuda")
    got = [B.paged_append(p, c.handle(p), x, x, q=t, positions=pos, inv_freq=freq, cu_new=cu) for t in (q, q.contiguous())]
    assert got[0].is_contiguous() and torch.equal(*got)


def test_append_with_its_output_beside_and_over_what_it_reads():
    """The rotated queries may go between the tokens of one projection's output, not over its parts."""
    p, n = _params(4, 2, 64, BF16), 3
    c = Cache([2, 1], 2, 64, 16, BF16, fill=0.0)
    wide = c.randn(n, 8 * 64 + n * 4 * 64)                             # queries, keys and values of a token, then room for all queries
    parts = [wide[:, 64 * a:64 * b].unflatten(1, (b - a, 64)) for a, b in ((0, 4), (4, 6), (6, 8))]
    freq, cu = torch.linspace(1.0, 0.001, 32, device="cuda"), torch.tensor([0, 2, 3], dtype=torch.int32, device="cuda")
    kw = dict(inv_freq=freq, cu_new=cu, positions=torch.arange(n, dtype=torch.int32, device="cuda") * 5)
    ref = B.paged_append(p, c.handle(p), parts[1], parts[2], q=parts[0], **kw)
    before = wide[:, :8 * 64].clone()
    for row in range(n):
        gap = wide[row, 8 * 64:].view(n, 4, 64)
        assert torch.equal(B.paged_append(p, c.handle(p), parts[1], parts[2], q=parts[0], q_out=gap, **kw), ref)
    for start in (0, 5 * 64, 7 * 64, 8 * 64 + 64):                     # the last one begins in the room and ends in the next token
        with pytest.raises(B.SablockError):
            B.paged_append(p, c.handle(p), parts[1], parts[2], q=parts[0], q_out=wide.flatten()[start:start + n * 256].view(n, 4, 64), **kw)
    assert torch.equal(wide[:, :8 * 64], before)
