"""Low-rank adapters of many requests (csb_adapter_add) against the formula in 64 bits on the host.

Tolerance: A X sums `cols` products (exact for 16-bit operands), B (A X) sums up to `rank`; in any order both sums are
within n 2^-24 of the sum of their absolute values: with S the formula over absolute values (Y's own among them),
(cols + rank + 6) 2^-24 S bounds an entry's error."""
import math
import sys

import numpy as np
import pytest
import torch

import lm_reference as ref
from paper_2005_05758_amd import CsbMatrix, adapter_add, VAL_BF16
from paper_2005_05758_amd.binding import lib

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda") if x is not None else None


def check(fmt, rows, cols, lengths, n, rank, ids, ranks=None, scales=True, batch=None, starts=True, ldx=None, ldy=None, shift=0, seed=0):
    batch = batch or sum(lengths)
    say(f"[adapter] {fmt} {rows}x{cols} batch {batch} lengths={lengths[:12]} rank {rank} ids={ids[:12]} ranks={ranks} ldx={ldx} ldy={ldy} shift={shift}")
    t = torch.Generator().manual_seed(seed)
    typ = TYPES[fmt]
    rnd = lambda *s: torch.randn(*s, generator=t)        # noqa: E731
    X, Y = rnd(cols, batch).to(typ), rnd(rows, batch)
    A, B = (rnd(n, rank, cols) * cols ** -0.5).to(typ), (rnd(n, rows, rank) * 0.2).to(typ)
    sc = rnd(n) if scales else None

    def placed(x, ld):
        """x in rows of ld elements (NaN between them), its base `shift` elements off."""
        flat = torch.full((x.shape[0] * ld + shift,), math.nan, dtype=x.dtype, device="cuda")[shift:]
        view = flat.view(x.shape[0], ld)[:, :x.shape[1]]
        view.copy_(x)
        return view
    Xd, Yd = placed(X, ldx or batch), placed(Y, ldy or batch)
    Ad, Bd = (placed(x.reshape(1, -1), x.numel()).view(x.shape) for x in (A, B))
    if ranks is not None:                                # what is stored past an adapter's rank is not read
        for a, r in enumerate(ranks):
            Ad[a, max(r, 0):] = math.nan
            Bd[a, :, max(r, 0):] = math.nan
    first = np.concatenate([[0], np.cumsum(lengths)]).astype(int)
    ranges = [(first[i], first[i + 1]) for i in range(len(lengths))]
    got = adapter_add(Yd, Xd, Ad, Bd, i32(ids), starts=i32(list(first)) if starts else None, scales=sc.cuda() if scales else None, ranks=i32(ranks))
    torch.cuda.synchronize()
    assert got is Yd
    args = [ref.widen(x) for x in (Y, X, A, B)] + [ranges, ids, ref.widen(sc) if scales else np.ones(n), ranks if ranks is not None else [rank] * n]
    want, size = ref.adapters(*args), ref.adapter_sizes(*args)
    y = Yd.cpu().double().numpy()
    far = np.abs(y - want) - (cols + rank + 6) * 2.0 ** -24 * size
    assert far.max() <= 0, far.max()
    same = np.ones(batch, bool)
    for (f, e), a in zip(ranges, ids):
        if 0 <= a < n:
            same[f:e] = False
    assert np.array_equal(y[:, same], Y.double().numpy()[:, same])


@pytest.mark.parametrize("fmt", sorted(TYPES))
@pytest.mark.parametrize("rows,cols,lengths,n,rank", [
    (1, 1, [1], 1, 1), (64, 32, [1, 1, 1], 2, 16), (130, 665, [33, 1, 65], 2, 8), (513, 153, [5, 0, 32, 31, 0, 64, 2], 3, 5),
    (100, 72, [40], 1, 33), (257, 1000, [7, 90], 2, 64), (65, 130, [20, 21, 22], 3, 128), (70, 2049, [3, 30], 2, 100)])
def test_shapes(fmt, rows, cols, lengths, n, rank):
    g = np.random.default_rng(rows)
    ids = [int(x) for x in g.integers(0, n, len(lengths))]
    check(fmt, rows, cols, lengths, n, rank, ids, seed=rows)
    if len(ids) > 1:
        ids[0], ids[-1] = -1, n                          # no adapter
    check(fmt, rows, cols, lengths, n, rank, ids, ranks=[int(x) for x in g.integers(0, rank + 1, n)], scales=False, seed=rows + 1)


@pytest.mark.parametrize("fmt", sorted(TYPES))
def test_one_column_each(fmt):
    g = np.random.default_rng(4)
    ids = [int(x) for x in g.integers(-1, 9, 70)]
    check(fmt, 200, 320, [1] * 70, 9, 16, ids, starts=False)
    check(fmt, 200, 320, [1] * 70, 9, 16, ids)
    check(fmt, 8, 4096, [1], 1, 16, [0], starts=False)


@pytest.mark.parametrize("fmt", sorted(TYPES))
@pytest.mark.parametrize("rank", [16, 64, 128])
def test_long_requests(fmt, rank):
    """Requests of many columns, aligned operands; one long one behind short ones that share its first tile."""
    check(fmt, 200, 1024, [70, 130], 2, rank, [1, 0], ranks=[rank, rank // 2], seed=rank)
    check(fmt, 72, 512, [1] * 9 + [1999], 6, rank, [0, 1, 2, 3, 4, 5, 0, -1, 1, 3], seed=rank + 1)


@pytest.mark.parametrize("fmt", sorted(TYPES))
@pytest.mark.parametrize("rank", [24, 64])
def test_short_requests_of_many_ranks(fmt, rank):
    """Several adapters in a tile, aligned operands and others, columns of the projection that end inside a step."""
    check(fmt, 130, 1048, [5, 9, 30, 1, 16, 3], 4, rank, [3, 0, 2, 3, 1, -1], ranks=[rank, 3, rank - 1, rank // 2], seed=rank)
    check(fmt, 130, 1047, [5, 9, 3, 1, 6, 3], 4, rank, [3, 0, 2, 3, 1, -1], ranks=[rank, 3, rank - 1, rank // 2], seed=rank)


def test_tall():
    """More rows than a launch's second dimension has workgroups of 16 for."""
    check("bf16", 16 * 65535 + 70, 8, [1, 1], 2, 8, [1, 0])


def test_many_requests():
    g = np.random.default_rng(5)
    lengths = [int(x) for x in g.integers(0, 3, 600)]
    check("bf16", 48, 64, lengths, 20, 4, [int(x) for x in g.integers(-1, 20, 600)])


@pytest.mark.parametrize("fmt", sorted(TYPES))
def test_strides_and_alignment(fmt):
    for ldx, ldy, shift in ((50, 47, 0), (51, 64, 0), (64, 51, 1), (48, 48, 2), (96, 47, 3)):
        check(fmt, 96, 160, [20, 27], 2, 16, [1, 0], ldx=ldx, ldy=ldy, shift=shift)
    check(fmt, 40, 64, [10, 20], 2, 8, [1, 0], batch=47)  # columns that no request has


def test_not_finite():
    """What is not finite in a column of X changes that column of Y only; columns without an adapter are not read."""
    X = torch.randn(256, 40, device="cuda").bfloat16()
    A, B = torch.randn(2, 16, 256, device="cuda").bfloat16(), torch.randn(2, 100, 16, device="cuda").bfloat16()
    Y = torch.randn(100, 40, device="cuda")
    ids, starts = i32([0, -1, 1]), i32([0, 10, 20, 40])
    clean = adapter_add(Y.clone(), X, A, B, ids, starts=starts)
    for j, n, x in ((3, 4, math.inf), (100, 5, math.nan), (7, 11, math.nan), (255, 39, -math.inf)):
        X[j, n] = x
    got = adapter_add(Y.clone(), X, A, B, ids, starts=starts)
    torch.cuda.synchronize()
    hit = [4, 5, 39]
    rest = [n for n in range(40) if n not in hit]
    assert torch.equal(got[:, rest], clean[:, rest]) and not torch.isfinite(got[:, hit]).any()


def test_beside_a_pruned_projection():
    """csb_spmm_bfloat's result and the adapters of its requests on top."""
    g = np.random.default_rng(6)
    W = (g.normal(0, 0.05, (256, 192)) * (g.random((256, 1)) < 0.5) * (g.random((1, 192)) < 0.5)).astype(np.float32)
    M = CsbMatrix(W, 32, 32)
    M.set_value_format(VAL_BF16)
    M.plan()
    M.upload()
    X = torch.randn(192, 64, device="cuda").bfloat16()
    A, B = torch.randn(3, 8, 192, device="cuda").bfloat16(), torch.randn(3, 256, 8, device="cuda").bfloat16()
    ids, starts = [2, -1, 0], [0, 20, 30, 64]
    Y = M.spmm_bfloat(X)
    base = Y.clone()
    adapter_add(Y, X, A, B, i32(ids), starts=i32(starts))
    torch.cuda.synchronize()
    args = [ref.widen(x) for x in (base, X, A, B)] + [[(0, 20), (20, 30), (30, 64)], ids, np.ones(3), [8] * 3]
    assert (np.abs(ref.widen(Y) - ref.adapters(*args)) <= 206 * 2.0 ** -24 * ref.adapter_sizes(*args)).all()
    assert torch.equal(Y[:, 20:30], base[:, 20:30])


def test_stream_graph_and_repeats():
    X, Y0 = torch.randn(640, 77, device="cuda").half(), torch.randn(300, 77, device="cuda")
    A, B = torch.randn(4, 16, 640, device="cuda").half(), torch.randn(4, 300, 16, device="cuda").half()
    ids, starts = i32([3, 1, 0]), i32([0, 33, 34, 77])
    Y = Y0.clone()
    torch.cuda.synchronize()

    def once(stream=None):
        y = Y0.clone()
        torch.cuda.synchronize()
        adapter_add(y, X, A, B, ids, starts=starts, stream=stream)
        torch.cuda.synchronize()
        return y
    want = once()
    assert torch.equal(once(), want) and torch.equal(once(torch.cuda.Stream()), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        adapter_add(Y, X, A, B, ids, starts=starts)
    for _ in range(3):
        X.copy_(torch.randn_like(X))
        want = once()
        Y.copy_(Y0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, want)


def test_offsets_past_32_bits():
    """Rows of X and Y further apart than 2^31 elements in all."""
    ld = 2 ** 31 // 600
    X, Y = (torch.empty(700, ld, dtype=d, device="cuda") for d in (torch.bfloat16, torch.float32))
    A, B = torch.randn(1, 4, 700, device="cuda").bfloat16(), torch.randn(1, 700, 4, device="cuda").bfloat16()
    x, y = torch.randn(700, 33, device="cuda").bfloat16(), torch.randn(700, 33, device="cuda")
    X[:, :33], Y[:, :33] = x, y
    ids, starts = i32([0]), i32([0, 33])
    adapter_add(Y[:, :33], X[:, :33], A, B, ids, starts=starts)
    adapter_add(y, x, A, B, ids, starts=starts)
    torch.cuda.synchronize()
    assert torch.equal(Y[:, :33], y)


def test_offsets_out_of_range_stay_inside():
    X, A, B = torch.randn(64, 40, device="cuda"), torch.randn(2, 4, 64, device="cuda"), torch.randn(2, 30, 4, device="cuda")
    ys = [adapter_add(torch.zeros(30, 40, device="cuda"), X, A, B, i32([0, 1]), starts=i32(s)) for s in ([-9, 20, 10 ** 6], [0, 20, 40])]
    torch.cuda.synchronize()
    assert torch.equal(*ys)


def test_refusals():
    X, Y = torch.zeros(64, 8, device="cuda"), torch.zeros(32, 8, device="cuda")
    A, B = torch.zeros(2, 4, 64, device="cuda"), torch.zeros(2, 32, 4, device="cuda")
    ids, ws = i32([0] * 8), torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    names = "type X ldx Y ldy rows cols batch A B n rank d_rank scale n_seg start id ws stream".split()
    good = dict(zip(names, [0, X.data_ptr(), 8, Y.data_ptr(), 8, 32, 64, 8, A.data_ptr(), B.data_ptr(), 2, 4, None, None, 8, None, ids.data_ptr(),
                            ws.data_ptr(), None]))

    def call(**change):
        return lib().csb_adapter_add(*({**good, **change}[n] for n in names))
    assert lib().csb_adapter_workspace_bytes(64, 8, 8, 4) <= ws.numel()
    assert call() == 0 and call(batch=0, n_seg=0) == 0
    for change in (dict(type=-1), dict(X=None), dict(Y=None), dict(A=None), dict(B=None), dict(id=None), dict(ws=None), dict(ldx=7), dict(ldy=7),
                   dict(rows=0), dict(cols=0), dict(batch=-1), dict(n=0), dict(rank=0), dict(n_seg=7), dict(n_seg=-1), dict(ws=ws.data_ptr() + 16),
                   dict(X=X.data_ptr() + 2), dict(Y=Y.data_ptr() + 1)):
        assert call(**change) == -1, change
    assert call(rank=129) == -4 and call(batch=(1 << 30) + 1, n_seg=(1 << 30) + 1, ldx=1 << 31, ldy=1 << 31) == -4
    with pytest.raises(AssertionError):
        adapter_add(Y, X.half(), A, B, ids)
    with pytest.raises(AssertionError):
        adapter_add(Y, X, A, B[:, :31], ids)
    torch.cuda.synchronize()


def test_refusals_of_sizes():
    X, Y = torch.zeros(64, 8, device="cuda"), torch.zeros(32, 8, device="cuda")
    A, B = torch.zeros(2, 4, 64, device="cuda"), torch.zeros(2, 32, 4, device="cuda")
    ids, ws = i32([0] * 8), torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    for rows, cols in ((1 << 31, 64), (32, 1 << 31), (1 << 62, 64)):
        assert lib().csb_adapter_add(0, X.data_ptr(), 8, Y.data_ptr(), 8, rows, cols, 8, A.data_ptr(), B.data_ptr(), 2, 4, None, None, 8, None,
                                     ids.data_ptr(), ws.data_ptr(), None) == -4
    torch.cuda.synchronize()
