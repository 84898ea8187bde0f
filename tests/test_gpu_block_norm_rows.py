"""Forward passes of more rows than one dimension of a grid has threads for."""
import pytest
import torch

import block_ref as ref
from paper_2309_03824_amd import binding as lrd

pytestmark = pytest.mark.gpu


def test_more_short_rows_than_one_dimension_of_a_grid():
    """2^26 rows of a wave each: the rows of the whole call are those of calls on parts, the last ones right."""
    d, T, k = 8, 2**26 + 5, 300
    g = torch.Generator(device="cuda").manual_seed(1)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    F, X = torch.randn(T, d, generator=g, **bf), torch.randn(T, d, generator=g, **bf)
    w = torch.rand(d, device="cuda", generator=g) + 0.5
    opt = lrd.BlockNorm(kind=lrd.NORM_LAYER, branch_scale=0.5)
    Y, N = torch.full_like(X, 9.0), torch.full_like(X, 9.0)
    lrd.block_norm_fwd(F, X, w, None, None, w, None, None, Y, N, opt)
    o = dict(layer=True, eps=float(torch.tensor(1e-5)), alpha=1.0, beta=0.5, gate_rows=0)
    y, n = ref.block_norm_fwd(F[-k:].cpu().double(), X[-k:].cpu().double(), w.cpu().double(), None, None, w.cpu().double(), None, None, o)
    ref.assert_close(Y[-k:], y, torch.bfloat16, "Y")
    ref.assert_close(N[-k:], n, torch.bfloat16, "N")
    part = 2**24 + 1
    for at in range(0, T, part):
        rows = slice(at, min(at + part, T))
        y, n = torch.empty_like(X[rows]), torch.empty_like(X[rows])
        lrd.block_norm_fwd(F[rows], X[rows], w, None, None, w, None, None, y, n, opt)
        assert torch.equal(Y[rows], y) and torch.equal(N[rows], n), at


def test_more_wide_rows_than_one_dimension_of_a_grid():
    """2^24 rows of 256 threads each, in their place: one row many times, the last ones others."""
    d, T, k = 1032, 2**24 + 3, 64
    X = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    row, last = (torch.randn(n, d, dtype=torch.bfloat16, device="cuda", generator=g) for n in (1, k))
    X.copy_(row.expand(T, d))
    X[-k:] = last
    w = torch.ones(d, device="cuda")
    lrd.block_norm_fwd(None, X, None, None, None, w, None, None, None, X, lrd.BlockNorm())
    o = dict(layer=False, eps=float(torch.tensor(1e-5)), alpha=1.0, beta=1.0, gate_rows=0)
    for got, x in ((X[-k:], last), (X[:1], row)):
        ref.assert_close(got, ref.block_norm_fwd(None, x.cpu().double(), None, None, None, w.cpu().double(), None, None, o)[1], torch.bfloat16, "N")
    for part in X[:-k].split(2**22):
        assert (part == X[0]).all()
