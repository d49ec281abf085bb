"""Views as operands of the language-model operators: those whose rows overlap are refused, those of one row or column are taken whatever
strides torch gives them."""
import sys

import pytest
import torch

import lm_reference as ref
from paper_2005_05758_amd import adapter_add, delta_recurrent, verify_drafts
from paper_2005_05758_amd.binding import CsbError

pytestmark = pytest.mark.gpu


def say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def adapters(rows, cols, batch, rank=4):
    t = torch.Generator().manual_seed(rows + cols)
    rnd = lambda *s: torch.randn(*s, generator=t).cuda()     # noqa: E731
    return rnd(rows, batch), rnd(cols, batch), rnd(1, rank, cols), rnd(1, rows, rank)


def test_rows_that_overlap_are_refused():
    """A row repeated, a window that slides over a signal: their strides are below a row's width.  Nothing is launched."""
    say("[views] refused")
    Y, X, A, B = adapters(24, 32, 16)
    ids, starts, before = i32([0]), i32([0, 16]), Y.clone()
    signal = torch.randn(32 + 15, device="cuda")
    for bad in (X[:1].expand(32, 16), signal.as_strided((32, 16), (1, 1)), X.flatten().as_strided((32, 16), (15, 1))):
        with pytest.raises(CsbError, match="leading dimension"):
            adapter_add(Y, bad, A, B, ids, starts=starts)
    for bad in (Y[:1].expand(24, 16), signal.as_strided((24, 16), (1, 1))):
        with pytest.raises(CsbError, match="leading dimension"):
            adapter_add(bad, X, A, B, ids, starts=starts)
    with pytest.raises(CsbError, match="leading dimension"):
        adapter_add(Y[:, :1], X[:1, :1].expand(32, 1), A, B, ids, starts=i32([0, 1]))
    q = torch.randn(1, 1, 8, device="cuda").expand(6, 1, 8)
    k, v, g = torch.randn(6, 1, 8, device="cuda"), torch.randn(6, 1, 8, device="cuda"), torch.zeros(6, 1, device="cuda")
    with pytest.raises(CsbError, match="leading dimension"):
        delta_recurrent(q, k, v, g, g)
    p = torch.softmax(torch.randn(1, 1, 50, device="cuda"), -1)
    for bad in (p.expand(2, 3, 50), p.expand(2, 1, 50)):
        n = bad.shape[1] - 1
        with pytest.raises((CsbError, AssertionError)):
            verify_drafts(bad, None, torch.zeros(2, n, dtype=torch.int32, device="cuda"), torch.zeros(2, n, device="cuda"), torch.zeros(2, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(Y, before)


@pytest.mark.parametrize("rows,cols,batch", [(1, 1, 5), (1, 32, 5), (24, 1, 5), (24, 32, 1), (1, 1, 1)])
def test_one_row_or_column(rows, cols, batch):
    """Parts of larger matrices, and rows of one that torch says nothing about."""
    say(f"[views] {rows}x{cols}, {batch} columns")
    Y, X, A, B = adapters(rows, cols, batch)
    want = torch.from_numpy(ref.adapters(*(ref.widen(x) for x in (Y, X, A, B)), [(0, batch)], [0], [1.0], [4]))
    wide_x, wide_y = torch.randn(cols, batch + 9, device="cuda"), torch.randn(rows, batch + 3, device="cuda")
    wide_x[:, 2:2 + batch], wide_y[:, 1:1 + batch] = X, Y
    pairs = [(X, Y), (wide_x[:, 2:2 + batch], wide_y[:, 1:1 + batch])]
    if cols == 1:
        pairs.append((X[0].expand(1, batch), Y.clone()))     # stride 0 of the one row
        pairs.append((X.as_strided((1, batch), (0, 1)), Y.clone()))
    if batch == 1:
        pairs.append((X.t().contiguous().t(), Y.t().contiguous().t()))
    for x, y in pairs:
        got = adapter_add(y.clone(memory_format=torch.preserve_format) if y is Y else y, x, A, B, i32([0]), starts=i32([0, batch]))
        torch.cuda.synchronize()
        assert (got.cpu().double() - want).abs().max() <= 1e-5 * max(1.0, want.abs().max())
