"""The 64-bit forms that the GPU tests of the block operators compare with: the generator against its authors' vectors, gradients
against differences; and the refusals of the entry points, which need no GPU."""
import ctypes

import numpy as np
import pytest
import torch

import block_ref as ref
from paper_2309_03824_amd import binding as lrd

D64 = torch.float64


def test_philox_known_answers():
    # test vectors published with the generator (philox4x32, 10 rounds)
    rows = [((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
            ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
            ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))]
    for ctr, key, want in rows:
        assert tuple(int(v) for v in ref.philox4x32(np.array([ctr], dtype=np.uint64), key)[0]) == want


@pytest.mark.parametrize("p", [0.1, 0.5, 0.9])
def test_dropout_keeps_its_share_and_its_mean(p):
    n = 1 << 18
    f = ref.drop_factors(n, p, 12345, 7)
    kept = float((f != 0).double().mean())
    assert abs(kept - (1 - p)) < 6 * (p * (1 - p) / n) ** 0.5 + 2 ** -17
    other = ref.drop_factors(n, p, 12345, 8)
    both = float(((f != 0) & (other != 0)).double().mean())
    assert abs(both - (1 - p) ** 2) < 6 * 0.5 / n ** 0.5
    # any piece of the array has the bits of the whole
    assert torch.equal(ref.drop_factors(1000, p, 12345, 7, first=4321), f[4321:5321])


def _difference(fn, x, direction, h=1e-5):
    return (fn(x + h * direction) - fn(x - h * direction)) / (2 * h)


@pytest.mark.parametrize("act", [0, 1, 2])
def test_gated_gradients_against_differences(act):
    g = torch.Generator().manual_seed(act)
    T, r, out = 5, 3, 7
    H, Uc, bias, dA = (torch.randn(*s, generator=g, dtype=D64) for s in ((T, 2 * r), (2, out, r), (2, out), (T, out)))
    (dzg, _), (dzu, _) = ref.gated(H, Uc, bias, act, torch.float32, dA)
    loss = lambda h, u, b: (dA * ref.gated(h, u, b, act, torch.float32)[0]).sum()
    for x, grad, fn in ((H, torch.cat((dzg @ Uc[0], dzu @ Uc[1]), 1), lambda v: loss(v, Uc, bias)),
                        (Uc, torch.stack((dzg.t() @ H[:, :r], dzu.t() @ H[:, r:])), lambda v: loss(H, v, bias)),
                        (bias, torch.stack((dzg.sum(0), dzu.sum(0))), lambda v: loss(H, Uc, v))):
        for _ in range(3):
            d = torch.randn(x.shape, generator=g, dtype=D64)
            assert abs(float(_difference(fn, x, d) - (grad * d).sum())) < 1e-7 * float((grad * d).abs().sum() + 1)


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("gate_rows", [0, 1, 3])
@pytest.mark.parametrize("post", [False, True])
def test_block_norm_gradients_against_differences(layer, gate_rows, post):
    g = torch.Generator().manual_seed(7)
    T, d = 7, 11
    o = dict(layer=layer, eps=1e-5, alpha=1.25, beta=0.75, gate_rows=gate_rows)
    rand = lambda *s: torch.randn(*s, generator=g, dtype=D64)
    at = dict(F=rand(T, d), X=rand(T, d), w_post=rand(d), b_post=rand(d), gate=rand(-(-T // (gate_rows or T)), d), w_pre=rand(d), b_pre=rand(d))
    if not post:
        at["w_post"] = at["b_post"] = None
    dY, dN, factors = rand(T, d), rand(T, d), ref.drop_factors(T * d, 0.3, 5, 6).reshape(T, d)

    def loss(**kw):
        a = dict(at, **kw)
        y, n = ref.block_norm_fwd(a["F"], a["X"], a["w_post"], a["b_post"], a["gate"], a["w_pre"], a["b_pre"], factors, o)
        return (dY * y[0]).sum() + (dN * n[0]).sum()

    (Y, _), _ = ref.block_norm_fwd(at["F"], at["X"], at["w_post"], at["b_post"], at["gate"], at["w_pre"], at["b_pre"], factors, o)
    grads = ref.block_norm_bwd(dY, dN, at["F"], Y, at["w_post"], at["b_post"], at["gate"], at["w_pre"], factors, o)
    for k, v in at.items():
        if v is None:
            assert "d" + k not in grads
            continue
        grad, direction = grads["d" + k][0], rand(*v.shape)
        got = _difference(lambda x: loss(**{k: x}), v, direction)
        assert abs(float(got - (grad * direction).sum())) < 1e-6 * float((grad * direction).abs().sum() + 1), k


# ------------------------------------------------------------------------------------------ refusals (nothing is launched)
P = 4096      # a fake, 16-byte aligned, never dereferenced address


def _call(fn, names, base, **kw):
    a = dict(zip(names, base), **kw)
    assert set(a) == set(names)
    return fn(*(a[n] for n in names))


def test_gated_refusals():
    names = ["X", "V", "U", "b", "A", "H", "act", "T", "n_in", "n_out", "r", "dt", "ws", "wsb", "st"]
    fwd = lambda **kw: _call(lrd._lib.lrd_linear_gated_fwd, names, [P, P, P, None, P, None, lrd.ACT_SILU, 8, 8, 8, 4, lrd.BF16, None, 0, None], **kw)
    for bad in (dict(X=None), dict(V=None), dict(U=None), dict(A=None), dict(T=0), dict(T=-1), dict(T=1 << 31), dict(n_in=0), dict(n_out=0), dict(r=0),
                dict(r=9), dict(act=3), dict(act=-1), dict(dt=2)):
        assert fwd(**bad) == lrd.ERR_INVALID_ARG, bad
    for bad in (dict(X=P + 2), dict(H=P + 8), dict(b=P + 4), dict(A=P + 1), dict(ws=P + 8, wsb=1 << 20)):
        assert fwd(**bad) == lrd.ERR_ALIGNMENT, bad
    assert fwd() == lrd.ERR_WORKSPACE                    # H has to go somewhere
    assert fwd(H=P, r=5) == lrd.ERR_WORKSPACE            # a raw rank: padded copies
    need = lrd.linear_gated_workspace_bytes(8, 8, 8, 4, lrd.BF16)
    assert need > 0 and fwd(ws=P, wsb=16) == lrd.ERR_WORKSPACE
    assert lrd.linear_gated_workspace_bytes(8, 8, 8, 9, lrd.BF16) == 0

    names = ["dA", "X", "H", "V", "U", "b", "dX", "dV", "dU", "db", "mask", "act", "T", "n_in", "n_out", "r", "dt", "ws", "wsb", "st"]
    bwd = lambda **kw: _call(lrd._lib.lrd_linear_gated_bwd, names, [P] * 5 + [None, P, P, P, None, 0, lrd.ACT_GELU, 8, 8, 8, 4, lrd.BF16, None, 0, None], **kw)
    for bad in (dict(dA=None), dict(V=None), dict(U=None), dict(dV=None), dict(dU=None), dict(X=None), dict(X=None, H=None, mask=1), dict(mask=4), dict(act=7),
                dict(T=0), dict(r=9)):
        assert bwd(**bad) == lrd.ERR_INVALID_ARG, bad
    for bad in (dict(dA=P + 2), dict(dX=P + 8), dict(dU=P + 4), dict(db=P + 4), dict(H=P + 2)):
        assert bwd(**bad) == lrd.ERR_ALIGNMENT, bad
    assert bwd() == lrd.ERR_WORKSPACE and bwd(ws=P, wsb=256) == lrd.ERR_WORKSPACE
    assert bwd(mask=3, dX=None, dV=None, dU=None) == lrd.OK      # nothing is asked for

    names = ["dA", "H", "V", "U", "b", "dX", "dZ", "dH", "act", "T", "n_in", "n_out", "r", "dt", "ws", "wsb", "st"]
    data = lambda **kw: _call(lrd._lib.lrd_linear_gated_bwd_data, names, [P] * 4 + [None, P, P, P, 0, 8, 8, 8, 4, lrd.BF16, None, 0, None], **kw)
    for bad in (dict(dA=None), dict(H=None), dict(dZ=None), dict(dH=None), dict(V=None), dict(U=None), dict(act=9), dict(dt=5), dict(T=0)):
        assert data(**bad) == lrd.ERR_INVALID_ARG, bad
    assert data(dZ=P + 2) == lrd.ERR_ALIGNMENT
    assert data(r=5) == lrd.ERR_WORKSPACE


def test_block_norm_refusals():
    opt = lrd.BlockNorm(dropout_p=0.1)
    by = ctypes.byref
    names = ["F", "X", "wo", "bo", "g", "wi", "bi", "rng", "Y", "N", "opt", "T", "d", "dt", "st"]
    fwd = lambda **kw: _call(lrd._lib.lrd_block_norm_fwd, names, [P, P, P, P, P, P, P, P, P, 2 * P, by(opt), 8, 8, lrd.BF16, None], **kw)
    wrong = [lrd.BlockNorm(kind=2), lrd.BlockNorm(eps=-1.0), lrd.BlockNorm(eps=float("nan")), lrd.BlockNorm(residual_scale=float("inf")),
             lrd.BlockNorm(branch_scale=float("nan")), lrd.BlockNorm(gate_rows=-1), lrd.BlockNorm(dropout_p=-0.1), lrd.BlockNorm(dropout_p=1.1),
             lrd.BlockNorm(dropout_p=float("nan"))]
    for bad in [dict(X=None), dict(Y=None), dict(F=None, N=None), dict(wi=None), dict(rng=None), dict(wo=None), dict(N=P), dict(T=0), dict(T=1 << 31),
                dict(d=0), dict(dt=9), dict(opt=None)] + [dict(opt=by(w)) for w in wrong]:
        assert fwd(**bad) == lrd.ERR_INVALID_ARG, bad
    for bad in (dict(F=P + 2), dict(wo=P + 4), dict(rng=P + 8), dict(N=P + 2), dict(g=P + 4)):
        assert fwd(**bad) == lrd.ERR_ALIGNMENT, bad
    assert fwd(d=16385) == lrd.ERR_UNSUPPORTED

    names = ["dY", "dN", "F", "Y", "wo", "bo", "g", "wi", "rng", "dX", "dF", "dwo", "dbo", "dg", "dwi", "dbi", "opt", "T", "d", "dt", "ws", "wsb", "st"]
    base = [P] * 9 + [P, 2 * P] + [P] * 5 + [by(opt), 8, 8, lrd.BF16, None, 0, None]
    bwd = lambda **kw: _call(lrd._lib.lrd_block_norm_bwd, names, base, **kw)
    none = dict(dwo=None, dbo=None, dg=None, dwi=None, dbi=None)
    for bad in [dict(dY=None, dN=None), dict(Y=None), dict(wi=None), dict(F=None), dict(dN=None), dict(g=None), dict(wo=None, bo=None), dict(wo=None, dwo=None, dbo=None),
                dict(rng=None), dict(dF=P), dict(T=0), dict(opt=None)] + [dict(opt=by(w)) for w in wrong]:
        assert bwd(**bad) == lrd.ERR_INVALID_ARG, bad
    for bad in (dict(dY=P + 2), dict(dg=P + 4), dict(ws=P + 8), dict(dF=P + 2)):
        assert bwd(**bad) == lrd.ERR_ALIGNMENT, bad
    assert bwd(d=16385) == lrd.ERR_UNSUPPORTED
    assert bwd() == lrd.ERR_WORKSPACE and bwd(ws=P, wsb=64) == lrd.ERR_WORKSPACE
    assert bwd(**none, F=None) == lrd.ERR_INVALID_ARG       # dF needs F where there is a norm behind the block
    assert lrd.block_norm_workspace_bytes(0, 8) == 0 and lrd.block_norm_workspace_bytes(8, 16385) == 0


def test_dropout_refusals():
    f = lrd._lib.lrd_dropout
    assert f(None, P, 8, 0.5, P, lrd.BF16, None) == lrd.ERR_INVALID_ARG
    assert f(P, None, 8, 0.5, P, lrd.BF16, None) == lrd.ERR_INVALID_ARG
    assert f(P, P, -1, 0.5, P, lrd.BF16, None) == lrd.ERR_INVALID_ARG
    assert f(P, P, 8, 0.5, P, 7, None) == lrd.ERR_INVALID_ARG
    assert f(P, P, 8, 0.5, None, lrd.BF16, None) == lrd.ERR_INVALID_ARG
    for p in (-1e-9, 1.0000001, float("nan"), float("inf")):
        assert f(P, P, 8, p, P, lrd.BF16, None) == lrd.ERR_INVALID_ARG
    assert f(P + 2, P, 8, 0.5, P, lrd.BF16, None) == lrd.ERR_ALIGNMENT
    assert f(P, P, 8, 0.5, P + 8, lrd.BF16, None) == lrd.ERR_ALIGNMENT
    assert f(P, P, 0, 0.5, P, lrd.BF16, None) == lrd.OK       # nothing to do


def test_wrappers_refuse_other_types_and_shapes():
    x, w = torch.zeros(4, 8), torch.zeros(8)
    for bad in (lambda: lrd.dropout(x, torch.zeros(8, 4), 0.5, None), lambda: lrd.dropout(x, x, 0.5, torch.zeros(2)), lambda: lrd.dropout(x, x, 0.5, None),
                lambda: lrd.block_norm_fwd(None, x, None, None, None, w.double(), None, None, None, x, lrd.BlockNorm()),
                lambda: lrd.block_norm_fwd(x, x, None, None, torch.zeros(3, 8), w, None, None, x, x, lrd.BlockNorm(gate_rows=2)),
                lambda: lrd.linear_gated_fwd(x, torch.zeros(6, 8), torch.zeros(2, 5, 4), None, torch.zeros(4, 5), None, 0)):
        with pytest.raises(ValueError):
            bad()


def test_workspaces_never_fall():
    for d in (1, 768, 5000, 16384):
        sizes = [lrd.block_norm_workspace_bytes(T, d) for T in range(1, 1400)]
        assert sizes == sorted(sizes)
    for n_in, n_out, r in ((768, 2048, 192), (1000, 1024, 257), (64, 64, 8), (4096, 512, 100), (4096, 11008, 1024)):
        for dt in (lrd.BF16, lrd.F32):
            sizes = [lrd.linear_gated_workspace_bytes(T, n_in, n_out, r, dt) for T in list(range(1, 1400)) + list(range(1400, 18000, 37))]
            assert sizes == sorted(sizes)


def test_a_gated_pair_at_the_greatest_width_is_not_padded_past_it():
    """A group has fewer than 2^24 outputs a layer: a pair whose padded width would reach that is computed as it is, without padded copies."""
    out, r = 2**24 - 1, 8
    assert 0 < lrd.linear_gated_workspace_bytes(1, 8, out, r, lrd.BF16) < 2 * out * r * 2       # (the bytes of one padded copy of U)
    assert lrd.linear_gated_workspace_bytes(1, 8, out + 1, r, lrd.BF16) == 0


def test_a_gated_pair_whose_gradients_pass_32_bits_is_not_padded():
    """Cropping counts a layer's dU in 32 bits: past that a pair is computed at its own sizes."""
    T, n_in, out, r = 1, 1024, 2**22 + 1, 1024
    padded = 2 * (out + 7) * r * (2 + 4)                # copies of U and of dU
    assert 0 < lrd.linear_gated_workspace_bytes(T, n_in, out, r, lrd.BF16) < padded
