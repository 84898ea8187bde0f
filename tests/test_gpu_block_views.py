"""Operands and results 16 bytes into a buffer, as the calls allow: the bits are those of buffers of their own."""
import pytest
import torch

from parity import workspace
from paper_2309_03824_amd import binding as lrd

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def moved(t):
    """A copy of t that begins 16 bytes into its buffer, and no further power of two."""
    if t is None:
        return None
    skip = 16 // t.element_size()
    flat = torch.empty(t.numel() + 2 * skip, dtype=t.dtype, device="cuda")
    out = flat[skip:skip + t.numel()].view(t.shape)
    assert out.data_ptr() % 32 == 16
    return out.copy_(t)


@pytest.mark.parametrize("p", [0.0, 0.3])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 4096, 100003])
def test_dropout(n, dt, p):
    X = torch.randn(n, generator=torch.Generator().manual_seed(n)).to(TYPES[dt]).cuda()
    rng = torch.tensor([3, 5], dtype=torch.int64, device="cuda")
    Y, x = torch.empty_like(X), moved(X)
    lrd.dropout(X, Y, p, rng)
    y = moved(torch.zeros_like(X))
    lrd.dropout(x, y, p, moved(rng))
    assert torch.equal(y, Y) and torch.equal(x, X)
    lrd.dropout(x, x, p, rng)
    assert torch.equal(x, Y)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(5, 3), (9, 64), (40, 1001), (33, 2048), (6, 5003), (5, 16384)])
def test_block_norm(T, d, dt):
    td, g = TYPES[dt], torch.Generator().manual_seed(d)
    rand = lambda *s: torch.randn(*s, generator=g).cuda()
    opt = lrd.BlockNorm(kind=lrd.NORM_LAYER, dropout_p=0.2, gate_rows=4)
    F, X, dY, dN = (rand(T, d).to(td) for _ in range(4))
    w_post, b_post, w_pre, b_pre, gate = rand(d), rand(d), rand(d), rand(d), rand(-(-T // 4), d)
    rng = torch.tensor([3, 5], dtype=torch.int64, device="cuda")

    def step(at):
        f, x, y, n, wo, bo, wi, bi, gt = (at(t) for t in (F, X, torch.zeros_like(X), torch.zeros_like(X), w_post, b_post, w_pre, b_pre, gate))
        lrd.block_norm_fwd(f, x, wo, bo, gt, wi, bi, at(rng), y, n, opt)
        out = [at(torch.zeros_like(t)) for t in (X, X, w_post, b_post, gate, w_pre, b_pre)]
        ws = at(workspace(lrd.block_norm_workspace_bytes(T, d)))
        lrd.block_norm_bwd(at(dY), at(dN), f, y, wo, bo, gt, wi, at(rng), *out, opt, ws)
        return [y, n] + out
    for got, want in zip(step(moved), step(lambda t: t)):
        assert torch.equal(got, want)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,n_in,n_out,r", [(1, 64, 96, 24), (40, 64, 100, 31), (600, 256, 520, 64), (1500, 128, 1032, 40), (700, 600, 1000, 520), (300, 65, 67, 31)])
def test_gated(T, n_in, n_out, r, dt):
    r = min(r, n_in, n_out)
    td, g = TYPES[dt], torch.Generator().manual_seed(T)
    rand = lambda *s: (torch.randn(*s, generator=g) / s[-1] ** 0.5).to(td).cuda()
    X, V, Uc, dA, b = rand(T, n_in), rand(2 * r, n_in), rand(2, n_out, r), rand(T, n_out), torch.randn(2, n_out, generator=g).cuda()
    act = lrd.ACT_GELU

    def step(at):
        ws = at(workspace(lrd.linear_gated_workspace_bytes(T, n_in, n_out, r, lrd.BF16 if dt == "bf16" else lrd.F32)))
        x, v, u, da, bias = (at(t) for t in (X, V, Uc, dA, b))
        new = lambda *s, dtype=td: at(torch.zeros(*s, dtype=dtype, device="cuda"))
        A, H, dX, dZ, dH = new(T, n_out), new(T, 2 * r), new(T, n_in), new(2, T, n_out), new(T, 2 * r)
        lrd.linear_gated_fwd(x, v, u, bias, A, H, act, ws)
        lrd.linear_gated_bwd_data(da, H, v, u, bias, dX, dZ, dH, act, ws)
        f = torch.float32
        grads = [new(T, n_in), new(2 * r, n_in, dtype=f), new(2, n_out, r, dtype=f), new(2, n_out, dtype=f)]
        lrd.linear_gated_bwd(da, x, H, v, u, bias, *grads, 0, act, ws)
        return [A, H, dX, dZ, dH] + grads
    for got, want in zip(step(moved), step(lambda t: t)):
        assert torch.equal(got, want)
