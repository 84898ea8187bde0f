"""The pass between two blocks (norms, gate, dropout, residual sum), its backward, and dropout by itself, against 64 bits."""
import pytest
import torch

import block_ref as ref
from parity import workspace
from paper_2309_03824_amd import binding as lrd

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SEED, CALL = 0x1234567890abcdef, (1 << 40) + 5


def host(t):
    return None if t is None else t.cpu().double()


class Case:
    def __init__(self, T, d, dt, *, post=True, pre=True, bias=True, gate=True, gate_rows=0, p=0.0, layer=False, alpha=1.25, beta=0.75, seed=0):
        g = torch.Generator().manual_seed(seed + 31 * T + d)
        td = TYPES[dt]
        self.T, self.d, self.td = T, d, td
        act = lambda std=1.0, off=0.0: (torch.randn(T, d, generator=g) * std + off).to(td).cuda()
        par = lambda n=None: (torch.randn(*((n, d) if n else (d,)), generator=g) * 0.5 + 1).cuda()
        self.F, self.X, self.dY, self.dN = act(0.7), act(2.0, 0.5), act(), act() if pre else None
        self.w_post, self.b_post = (par() if post else None), (par() if post and bias else None)
        self.w_pre, self.b_pre = (par() if pre else None), (par() if pre and bias else None)
        self.gate = par(-(-T // (gate_rows or T))) if gate else None
        self.rng = torch.tensor([SEED, CALL], dtype=torch.int64, device="cuda") if p else None
        self.opt = lrd.BlockNorm(kind=lrd.NORM_LAYER if layer else lrd.NORM_RMS, eps=1e-5, residual_scale=alpha, branch_scale=beta, dropout_p=p, gate_rows=gate_rows)
        self.o = dict(layer=layer, eps=float(torch.tensor(1e-5)), alpha=alpha, beta=beta, gate_rows=gate_rows)
        self.factors = ref.drop_factors(T * d, p, SEED, CALL).reshape(T, d) if p else None

    def forward(self):
        Y, N = torch.empty_like(self.X), torch.empty_like(self.X) if self.w_pre is not None else None
        lrd.block_norm_fwd(self.F, self.X, self.w_post, self.b_post, self.gate, self.w_pre, self.b_pre, self.rng, Y, N, self.opt)
        return Y, N

    def check_forward(self):
        Y, N = self.forward()
        y, n = ref.block_norm_fwd(*(host(t) for t in (self.F, self.X, self.w_post, self.b_post, self.gate, self.w_pre, self.b_pre)), self.factors, self.o)
        ref.assert_close(Y, y, self.td, "Y")
        if N is not None:
            ref.assert_close(N, n, self.td, "N")
        return Y

    def backward(self, Y, ws=None):
        like = lambda t: None if t is None else torch.full_like(t, 9.0)
        out = dict(dX=torch.empty_like(self.X), dF=torch.empty_like(self.X), dw_post=like(self.w_post), db_post=like(self.b_post), dgate=like(self.gate),
                   dw_pre=like(self.w_pre), db_pre=like(self.b_pre))
        ws = ws if ws is not None else workspace(lrd.block_norm_workspace_bytes(self.T, self.d))
        lrd.block_norm_bwd(self.dY, self.dN, self.F, Y, self.w_post, self.b_post, self.gate, self.w_pre, self.rng, out["dX"], out["dF"], out["dw_post"],
                           out["db_post"], out["dgate"], out["dw_pre"], out["db_pre"], self.opt, ws)
        return out

    def check_backward(self, Y):
        out = self.backward(Y)
        want = ref.block_norm_bwd(*(host(t) for t in (self.dY, self.dN, self.F, Y, self.w_post, self.b_post, self.gate, self.w_pre)), self.factors, self.o)
        for k, v in out.items():
            if v is not None:
                ref.assert_close(v, want[k], self.td if k in ("dX", "dF") else torch.float32, k)
        return out


# widths around those at which a row goes to more threads, with and without whole 16-byte groups
WIDTHS = [1, 3, 8, 64, 100, 511, 512, 513, 768, 1000, 1024, 1028, 2048, 2056, 4095, 4096, 5000, 8192, 8200, 12289, 16384]


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", WIDTHS)
def test_widths(d, dt, layer):
    c = Case(37, d, dt, layer=layer, gate_rows=17, p=0.25)
    c.check_backward(c.check_forward())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [2, 4, 5, 7, 9, 10, 15, 17, 31, 255, 257, 505, 519, 1017, 1023, 1025, 1031, 2047, 2049, 2061, 2503, 4097, 8191, 8193, 16379, 16383])
def test_groups_that_end_with_their_row(d, dt):
    for T, gate_rows in ((1, 0), (11, 2), (300, 150)):
        c = Case(T, d, dt, layer=d % 2 == 0, gate_rows=gate_rows, p=0.25)
        c.check_backward(c.check_forward())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("T,gate_rows", [(1, 0), (1, 1), (2, 1), (9, 2), (33, 3), (100, 16), (100, 17), (700, 99), (700, 699), (1300, 1), (5000, 0), (5000, 2500), (9000, 4)])
@pytest.mark.parametrize("d", [96, 1032])
def test_tokens_and_gates(T, gate_rows, d, dt):
    c = Case(T, d, dt, gate_rows=gate_rows, layer=T % 2 == 0)
    c.check_backward(c.check_forward())


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("pre", [False, True])
@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("p", [0.0, 0.1])
@pytest.mark.parametrize("layer", [False, True])
def test_every_combination_of_parts(post, pre, gate, bias, p, layer):
    for dt, d in (("bf16", 264), ("f32", 1541), ("f32", 640)):
        c = Case(50, d, dt, post=post, pre=pre, gate=gate, bias=bias, p=p, gate_rows=20, layer=layer)
        c.check_backward(c.check_forward())


@pytest.mark.parametrize("p", [1e-7, 0.999, 1.0])
def test_nothing_or_everything_dropped(p):
    c = Case(21, 136, "bf16", p=p, gate_rows=4)
    c.check_backward(c.check_forward())


def test_a_gate_for_more_tokens_than_there_are():
    for rows in (50, 51, 1000):
        c = Case(50, 200, "bf16", gate_rows=rows, layer=True)
        c.check_backward(c.check_forward())


@pytest.mark.parametrize("d", [768, 4096, 16384])
def test_each_gradient_by_itself(d):
    """Whatever else a call asks for, each gradient has the same bits, and what it does not ask for is not written."""
    c = Case(150, d, "bf16", gate_rows=30, p=0.2, layer=True)
    Y, _ = c.forward()
    ws = workspace(lrd.block_norm_workspace_bytes(c.T, d))
    whole = c.backward(Y, ws)
    for k in whole:
        alone = torch.full_like(whole[k], 5.0)
        args = {n: None for n in whole}
        args[k] = alone
        need_f = k in ("dF", "dgate", "dw_post", "db_post")
        lrd.block_norm_bwd(c.dY, c.dN, c.F if need_f else None, Y, c.w_post, c.b_post, c.gate, c.w_pre, c.rng if need_f else None, args["dX"], args["dF"],
                           args["dw_post"], args["db_post"], args["dgate"], args["dw_pre"], args["db_pre"], c.opt, ws if k[1] != "X" and k != "dF" else None)
        assert torch.equal(alone, whole[k]), k


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [128, 513, 4096])
def test_first_norm_and_one_sided_gradients(dt, d):
    c = Case(45, d, dt, layer=True)
    N = torch.empty_like(c.X)
    lrd.block_norm_fwd(None, c.X, None, None, None, c.w_pre, c.b_pre, None, None, N, c.opt)
    o = dict(c.o, alpha=1.0)
    _, n = ref.block_norm_fwd(None, host(c.X), None, None, None, host(c.w_pre), host(c.b_pre), None, o)
    ref.assert_close(N, n, c.td, "N")
    ws = workspace(lrd.block_norm_workspace_bytes(c.T, d))
    opt = lrd.BlockNorm(kind=lrd.NORM_LAYER, eps=1e-5)
    for dY in (None, c.dY):
        dX, dw, db = torch.empty_like(c.X), torch.empty_like(c.w_pre), torch.empty_like(c.b_pre)
        lrd.block_norm_bwd(dY, c.dN, None, c.X, None, None, None, c.w_pre, None, dX, None, None, None, None, dw, db, opt, ws)
        want = ref.block_norm_bwd(host(dY), host(c.dN), None, host(c.X), None, None, None, host(c.w_pre), None, o)
        for got, k in ((dX, "dX"), (dw, "dw_pre"), (db, "db_pre")):
            ref.assert_close(got, want[k], c.td if k == "dX" else torch.float32, k)
    # past the last block: no norm follows
    c = Case(45, d, dt, pre=False, layer=True)
    c.check_backward(c.check_forward())


def test_rows_that_are_constant_tiny_or_far_from_zero():
    for layer in (False, True):
        c = Case(64, 640, "f32", layer=layer, gate=False)
        c.F[0], c.F[1], c.F[2] = 0.0, 3.0, 1e-12
        c.X[0], c.X[1], c.X[3], c.X[4] = 0.0, 7.0, 0.0, c.X[4] + 1000.0
        c.F[3] = 0.0
        c.F[5] += 300.0
        c.check_backward(c.check_forward())


def test_infinities_and_nan_stay_in_their_row_and_are_dropped_with_their_element():
    c = Case(6, 96, "bf16", post=False, pre=True, gate=False, bias=False, p=0.5)
    keep = c.factors != 0
    dropped = int((~keep[2]).nonzero()[0])
    c.F[2, dropped] = float("nan")
    c.F[3, int((~keep[3]).nonzero()[0])] = float("inf")
    c.F[4, int(keep[4].nonzero()[0])] = float("nan")
    Y, N = c.forward()
    assert torch.isfinite(Y[2:4].float()).all() and torch.isfinite(N[2:4].float()).all()
    assert int(torch.isnan(Y[4].float()).sum()) == 1 and torch.isnan(N[4].float()).all()
    assert torch.isfinite(Y[5].float()).all() and torch.isfinite(N[[0, 1, 5]].float()).all()


def test_results_in_the_place_of_operands():
    for d in (264, 515, 5000, 12304, 16001):
        c = Case(40, d, "bf16", p=0.1)
        Y, N = c.forward()
        x, f = c.X.clone(), c.F.clone()
        lrd.block_norm_fwd(f, x, c.w_post, c.b_post, c.gate, c.w_pre, c.b_pre, c.rng, x, f, c.opt)
        assert torch.equal(x, Y) and torch.equal(f, N)
        whole = c.backward(Y)
        dy, y = c.dY.clone(), Y.clone()
        like = lambda t: torch.empty_like(t)
        ws = workspace(lrd.block_norm_workspace_bytes(40, d))
        lrd.block_norm_bwd(dy, c.dN, c.F, y, c.w_post, c.b_post, c.gate, c.w_pre, c.rng, dy, y, like(c.w_post), like(c.b_post), like(c.gate), like(c.w_pre), like(c.b_pre),
                           c.opt, ws)
        assert torch.equal(dy, whole["dX"]) and torch.equal(y, whole["dF"])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [6, 264, 515, 2503, 4096, 9001, 12304])
def test_gradients_in_the_place_of_any_two_operands(d, dt):
    c = Case(40, d, dt, p=0.1, layer=True)
    Y, _ = c.forward()
    for with_n in (True, False):
        if not with_n:
            c.dN = None
        like = lambda t, there=True: torch.empty_like(t) if there else None
        ws = workspace(lrd.block_norm_workspace_bytes(40, d))

        def run(dY, dN, F, Y, dX, dF):
            sums = [like(c.w_post), like(c.b_post), like(c.gate), like(c.w_pre, with_n), like(c.b_pre, with_n)]
            lrd.block_norm_bwd(dY, dN, F, Y if with_n else None, c.w_post, c.b_post, c.gate, c.w_pre if with_n else None, c.rng, dX, dF, *sums, c.opt, ws)
            return [dX, dF] + [t for t in sums if t is not None]

        want = run(c.dY, c.dN, c.F, Y, torch.empty_like(Y), torch.empty_like(Y))
        at = ("dY", "dN", "F", "Y") if with_n else ("dY", "F")
        for a in at:
            for b in at:
                if a != b:
                    o = dict(dY=c.dY.clone(), dN=None if c.dN is None else c.dN.clone(), F=c.F.clone(), Y=Y.clone())
                    for x, y in zip(run(*o.values(), o[a], o[b]), want):
                        assert torch.equal(x, y), (a, b, with_n)


def test_rows_past_the_last_token_and_columns_past_a_row_are_left_alone():
    for d in (100, 1536):
        c = Case(13, d, "bf16", gate_rows=5)
        pad = 64
        big = lambda: torch.full((13 * d + pad,), 7.0, dtype=torch.bfloat16, device="cuda")
        y, n, dx, df = big(), big(), big(), big()
        view = lambda t: t[:13 * d].view(13, d)
        lrd.block_norm_fwd(c.F, c.X, c.w_post, c.b_post, c.gate, c.w_pre, c.b_pre, None, view(y), view(n), c.opt)
        g = torch.full((3 * d + pad,), 7.0, device="cuda")
        w = torch.full((d + pad,), 7.0, device="cuda")
        ws = workspace(lrd.block_norm_workspace_bytes(13, d))
        lrd.block_norm_bwd(c.dY, c.dN, c.F, view(y), c.w_post, c.b_post, c.gate, c.w_pre, None, view(dx), view(df), w[:d], None, g[:3 * d].view(3, d), None, None, c.opt, ws)
        for t, k in ((y, 13 * d), (n, 13 * d), (dx, 13 * d), (df, 13 * d), (g, 3 * d), (w, d)):
            assert (t[k:] == 7).all()


# ------------------------------------------------------------------------------------------ dropout by itself
def dropped(X, p, first=0):
    f = ref.drop_factors(X.numel(), p, SEED, CALL, first).to(torch.float32).reshape(X.shape)
    x = X.cpu().float()
    return torch.where(f != 0, x * f, torch.zeros_like(x)).to(X.dtype)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("p", [0.0, 1e-9, 0.1, 0.25, 0.5, 0.999, 1.0])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 2047, 4100 * 33, 1 << 20])
def test_dropout_bits(n, p, dt):
    X = torch.randn(n, generator=torch.Generator().manual_seed(n)).to(TYPES[dt]).cuda()
    rng = torch.tensor([SEED, CALL], dtype=torch.int64, device="cuda")
    flat = torch.full((n + 16,), 3.0, dtype=X.dtype, device="cuda")
    lrd.dropout(X, flat[:n], p, rng)
    assert torch.equal(flat[:n].cpu(), dropped(X, p)) and (flat[n:] == 3).all()
    lrd.dropout(X, X, p, rng if p > 1e-8 else None)
    assert torch.equal(X, flat[:n])


def test_dropout_of_an_array_past_32_bits():
    n = (1 << 31) + 13
    X = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    lrd.dropout(X, X, 0.3, torch.tensor([SEED, CALL], dtype=torch.int64, device="cuda"))
    for first in (0, (1 << 31) - 4096, n - 3000):
        got = X[first:first + 3000].cpu()
        assert torch.equal(got, dropped(torch.ones_like(got), 0.3, first))


def test_a_captured_step_goes_on_counting():
    """The generator's state is read at each replay: the masks of a captured step change with the call's number."""
    X, dY = torch.randn(300, 257).cuda(), torch.randn(300, 257).cuda()
    Y, dX = torch.empty_like(X), torch.empty_like(X)
    rng = torch.tensor([99, 0], dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lrd.dropout(X, Y, 0.4, rng)
        lrd.dropout(dY, dX, 0.4, rng)
        rng[1:].add_(1)
    rng.copy_(torch.tensor([99, 500], device="cuda"))
    last = None
    for rep in range(3):
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        f = ref.drop_factors(X.numel(), 0.4, 99, 500 + rep).float().reshape(X.shape).cuda()
        assert torch.equal(Y, X * f) and torch.equal(dX, dY * f)
        assert last is None or not torch.equal(last, f)
        last = f


def test_block_norm_replays():
    c = Case(600, 768, "bf16", gate_rows=200, p=0.1, layer=True)
    Y, N = torch.empty_like(c.X), torch.empty_like(c.X)
    ws = workspace(lrd.block_norm_workspace_bytes(600, 768))
    g = {k: torch.empty_like(v) for k, v in dict(dX=c.X, dF=c.X, dw_post=c.w_post, db_post=c.b_post, dgate=c.gate, dw_pre=c.w_pre, db_pre=c.b_pre).items()}

    def step():
        lrd.block_norm_fwd(c.F, c.X, c.w_post, c.b_post, c.gate, c.w_pre, c.b_pre, c.rng, Y, N, c.opt)
        lrd.block_norm_bwd(c.dY, c.dN, c.F, Y, c.w_post, c.b_post, c.gate, c.w_pre, c.rng, *g.values(), c.opt, ws)
    step()
    torch.cuda.synchronize()
    outs = [Y, N, *g.values()]
    want = [t.clone() for t in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for rep in range(3):
        for t in outs:
            t.fill_(float(rep))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, w) for t, w in zip(outs, want)), rep
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(t, w) for t, w in zip(outs, want)), rep


def test_rows_past_32_bits():
    """More than 2^31 elements: the last rows are those of a call on them alone."""
    d = 1024
    T = (1 << 31) // d + 300
    g = torch.Generator(device="cuda").manual_seed(3)
    F = torch.randn(T, d, device="cuda", dtype=torch.bfloat16, generator=g)
    X = torch.randn(T, d, device="cuda", dtype=torch.bfloat16, generator=g)
    gate = torch.randn(-(-T // 1000), d, device="cuda", generator=g)
    w = torch.rand(d, device="cuda", generator=g) + 0.5
    rng = torch.tensor([SEED, CALL], dtype=torch.int64, device="cuda")
    opt = lrd.BlockNorm(dropout_p=0.2, gate_rows=1000)
    Y, N = torch.empty_like(X), torch.empty_like(X)
    lrd.block_norm_fwd(F, X, w, None, gate, w, None, rng, Y, N, opt)
    at = (T - 1) // 1000 * 1000                      # the last group
    n = T - at
    factors = ref.drop_factors(n * d, 0.2, SEED, CALL, first=at * d).reshape(n, d)
    o = dict(layer=False, eps=float(torch.tensor(1e-5)), alpha=1.0, beta=1.0, gate_rows=0)
    y, nn = ref.block_norm_fwd(host(F[at:]), host(X[at:]), host(w), None, host(gate[-1:]), host(w), None, factors, o)
    ref.assert_close(Y[at:], y, torch.bfloat16, "Y")
    ref.assert_close(N[at:], nn, torch.bfloat16, "N")
    dX, dF, dgate = torch.empty_like(X), N, torch.empty_like(gate)
    ws = workspace(lrd.block_norm_workspace_bytes(T, d))
    lrd.block_norm_bwd(X, F, F, Y, w, None, gate, w, rng, dX, dF, None, None, dgate, None, None, opt, ws)
    want = ref.block_norm_bwd(host(X[at:]), host(F[at:]), host(F[at:]), host(Y[at:]), host(w), None, host(gate[-1:]), host(w), factors, o)
    ref.assert_close(dX[at:], want["dX"], torch.bfloat16, "dX")
    ref.assert_close(dF[at:], want["dF"], torch.bfloat16, "dF")
    ref.assert_close(dgate[-1:], want["dgate"], torch.float32, "dgate")
