"""The activations of the gated pairs over their range, tails included, relative to their value: with factors of single ones Zg is the input itself and Zu
is 1, so that A = act(z), dZu = act(z) and dZg = act'(z) for dA = 1, with one rounding and the activation's own error."""
import pytest
import torch

import block_ref as ref
from parity import workspace
from paper_2309_03824_amd import binding as lrd

pytestmark = pytest.mark.gpu
U = ref.U
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
CODE = {"bf16": lrd.BF16, "f32": lrd.F32}


def arguments(T, td):
    """T arguments: in bf16 every one of the type between 2^-20 and 13, both signs; then far ones and zero."""
    far = torch.tensor([0.0, -0.0, 13.5, -13.5, 20.0, -20.0, 60.0, -60.0, 1e4, -1e4, 1e30, -1e30])
    if td == torch.bfloat16:
        near = torch.arange(0x3580, 0x4151, dtype=torch.int16).view(torch.bfloat16).float()
        near = torch.cat((near, -near))
    else:
        near = torch.rand(T, generator=torch.Generator().manual_seed(3)) * 26 - 13
        near[::5] /= 16
    z = torch.cat((far, near))
    return z.repeat(-(-T // len(z)))[:T].to(td)


def normal_below(z):
    """The normal distribution, relative in its tail too (torch.special.ndtr is off by 1e-16 there, absolute)."""
    return torch.erfc(-z / 2 ** 0.5) / 2


def act_terms(z, act):
    if act != lrd.ACT_GELU:
        return ref.act_terms(z, act)
    below = normal_below(z)
    return z * below, below + z * torch.exp(-z * z / 2) / (2 * torch.pi) ** 0.5


def errors(z, act):
    """How far fp32 arithmetic may take act(z) and act'(z).
    GELU: Phi(-|z|) = exp(-z^2 / 2) g(t), t = 1 / (1 + 0.3 |z|): g's fit 1.7e-7; t off by four U, times |d ln g / d ln t| <= 2.7; its
    eight steps and rounded coefficients by eight U: 1.5e-6 at most.  The exponential: (0.75 z^2 + 2) 2^-23 by three roundings in its exponent.  SiLU: block_ref."""
    if act != lrd.ACT_GELU:
        return ref.act_errors(z, act, torch.float32)
    rel = 1.5e-6 + (0.75 * z * z + 2) * 2 * U
    tail, density = normal_below(-z.abs()), torch.exp(-z * z / 2) / (2 * torch.pi) ** 0.5
    a = act_terms(z, act)[0]
    return z.abs() * rel * tail + 2 * U * a.abs(), rel * (tail + z.abs() * density) + 4 * U * (normal_below(z) + z.abs() * density)


# input width, outputs, rank, tokens: one for each kernel of the second products and each number of its workgroups (16 x 16 blocks, 32 x 32 blocks, long
# batches, outputs off 8, any sizes)
KERNELS = [("bf16", 8, 8, 8, 4000), ("bf16", 8, 8, 8, 12000), ("bf16", 8, 8, 8, 20000), ("bf16", 8, 9, 8, 40000), ("bf16", 9, 9, 5, 40000), ("bf16", 8, 16, 3, 12000),
           ("f32", 8, 8, 8, 4000), ("f32", 8, 9, 5, 20000), ("f32", 8, 8, 8, 40000)]


@pytest.mark.parametrize("act", [lrd.ACT_NONE, lrd.ACT_GELU, lrd.ACT_SILU])
@pytest.mark.parametrize("dt,n_in,n_out,r,T", KERNELS)
def test_activation_relative_to_its_value(dt, n_in, n_out, r, T, act):
    td = TYPES[dt]
    z = arguments(T, td)
    X = torch.zeros(T, n_in, dtype=td)
    X[:, 0], X[:, 1] = z, 1
    V, Uc = torch.zeros(2 * r, n_in, dtype=td), torch.zeros(2, n_out, r, dtype=td)
    V[0, 0] = V[r, 1] = 1
    Uc[:, :, 0] = 1
    X, V, Uc = X.cuda(), V.cuda(), Uc.cuda()
    new = lambda *s: torch.empty(*s, dtype=td, device="cuda")
    A, H, dZ, dH = new(T, n_out), new(T, 2 * r), new(2, T, n_out), new(T, 2 * r)
    ws = workspace(lrd.linear_gated_workspace_bytes(T, n_in, n_out, r, CODE[dt]))
    lrd.linear_gated_fwd(X, V, Uc, None, A, H, act, ws)
    lrd.linear_gated_bwd_data(torch.ones_like(A), H, V, Uc, None, None, dZ, dH, act, ws)
    assert torch.equal(H[:, 0].cpu(), z) and (H[:, r] == 1).all()
    x = z.double()
    a, da = act_terms(x, act)
    far = x.abs() > 1e6                                # (z phi(z) in 64 bits too: 0, not infinity times 0)
    if act == lrd.ACT_GELU:
        da = torch.where(far, (x > 0).double(), da)
    if act == lrd.ACT_SILU:
        a, da = torch.where(far & (x < 0), torch.zeros_like(a), a), torch.where(far, (x > 0).double(), da)
    ea, eda = (torch.where(torch.isfinite(e), e, torch.zeros_like(e)) for e in errors(x, act))
    wide = lambda t: t[:, None].expand(T, n_out)
    for got, value, err, what in ((A, a, ea, "A"), (dZ[0], da, eda, "dZg"), (dZ[1], a, ea, "dZu")):
        ref.assert_close(got, (wide(value), wide(2 * err)), td, what)
