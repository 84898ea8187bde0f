"""The work by which the operators around the decomposed linears of a feed-forward block are judged:

  gated    two decomposed layers on one input, act(Zg) * Zu, as a gated feed-forward block begins: forward, or its backward;
  norm     what stands between two blocks: norm of the block's result, gate, dropout, residual sum, norm before the next block;
  dropout  by itself, with a counter-based generator whose mask is computed wherever it is needed.

A case is a dict of plain values.  H, dZ and dH are results in the type of the activations like every intermediate of a layer
pair: what follows starts from what is stored, here and in the library.
"""
import numpy as np
import torch

own = False

SEED_MIX = 0x5DEECE66D
ACTS = ("none", "gelu", "silu")
NORMS = ("rms", "layer")
TYPES = dict(bf16=torch.bfloat16, f32=torch.float32)


def listed():
    return [
        # Serving: one token through the gated half of a block.  Latency counts.
        dict(name="gated_token", op="gated", direction="infer", dtype="bf16", tokens=1, n_in=1024, n_out=4096, rank=256, act="silu", bias=False),
        # A ragged prompt through a layer at a rank straight from a compression ratio, before quantization.
        dict(name="gated_prompt_raw_rank", op="gated", direction="infer", dtype="bf16", tokens=509, n_in=768, n_out=2056, rank=193, act="gelu", bias=True),
        # A wide layer on a long batch, as prompts are taken in.
        dict(name="gated_prefill", op="gated", direction="infer", dtype="bf16", tokens=16384, n_in=4096, n_out=8192, rank=512, act="silu", bias=False),
        # The encoder's feed-forward sizes in training, forward: H is kept for the backward.
        dict(name="gated_train_forward", op="gated", direction="forward", dtype="bf16", tokens=8192, n_in=1024, n_out=4096, rank=256, act="silu", bias=True),
        # Its data gradient, as a stack's backward runs it: dZ and dH are kept for the weight gradients of all layers.
        dict(name="gated_train_data", op="gated", direction="data", dtype="bf16", tokens=8192, n_in=1024, n_out=4096, rank=256, act="silu", bias=True),
        # A single fp32 layer, all gradients in one call.
        dict(name="gated_f32", op="gated", direction="backward", dtype="f32", tokens=256, n_in=768, n_out=1536, rank=208, act="gelu", bias=True),
        # Serving: the norms around one token's block.
        dict(name="norm_token", op="norm", direction="forward", dtype="bf16", tokens=1, width=1024, kind="rms", post=True, pre=True, affine=False,
             gate_rows=0, gate=False, p=0.0, alpha=1.0, beta=1.0),
        # Training, adaptive gate of each sequence, dropout on the branch.
        dict(name="norm_train_forward", op="norm", direction="forward", dtype="bf16", tokens=8192, width=1024, kind="layer", post=True, pre=True, affine=True,
             gate_rows=512, gate=True, p=0.1, alpha=1.0, beta=1.0),
        dict(name="norm_train_backward", op="norm", direction="backward", dtype="bf16", tokens=8192, width=1024, kind="layer", post=True, pre=True,
             affine=True, gate_rows=512, gate=True, p=0.1, alpha=1.0, beta=1.0),
        # A wide stream in training, norm before the block only, learned scale of the branch.
        dict(name="norm_wide_backward", op="norm", direction="backward", dtype="bf16", tokens=16384, width=4096, kind="rms", post=False, pre=True,
             affine=False, gate_rows=0, gate=True, p=0.0, alpha=1.0, beta=0.5),
        # A short ragged batch of an odd width in fp32.
        dict(name="dropout_odd_f32", op="dropout", dtype="f32", tokens=509, width=1001, p=0.25),
        # Inside a block's feed-forward, at the encoder's sizes.
        dict(name="dropout_train", op="dropout", dtype="bf16", tokens=8192, width=4096, p=0.1),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(("gated", "gated", "gated", "norm", "norm", "dropout"))
    if op == "gated":
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        direction = rng.choice(("infer", "forward", "data", "backward"))
        n_in, n_out = rng.choice((512, 768, 1000, 1024, 2048)), rng.choice((512, 1001, 1536, 2056, 2730, 4096))
        r = rng.randint(min(n_in, n_out) // 6, min(min(n_in, n_out) // 2, 512))
        m = rng.choice((1, 16, 64, 64))
        return dict(op=op, direction=direction, dtype=dtype, tokens=_log(rng, 1, 8192 if dtype == "bf16" else 1024), n_in=n_in, n_out=n_out,
                    rank=max(m, r // m * m), act=rng.choice(ACTS[1:] + ("silu",)), bias=rng.random() < 0.5)
    if op == "norm":
        T = _log(rng, 1, 8192)
        post, pre = rng.choice(((True, True), (False, True), (True, False)))
        return dict(op=op, direction=rng.choice(("forward", "backward")), dtype=rng.choice(("bf16", "bf16", "f32")), tokens=T,
                    width=rng.choice((64, 511, 768, 1000, 1024, 1536, 2048, 4096)), kind=rng.choice(NORMS), post=post, pre=pre, affine=rng.random() < 0.5,
                    gate_rows=rng.choice((0, 0, _log(rng, 1, max(1, T)))), gate=rng.random() < 0.6, p=rng.choice((0.0, 0.1, 0.25)),
                    alpha=rng.choice((1.0, 1.5)), beta=rng.choice((1.0, 0.5)))
    return dict(op=op, dtype=rng.choice(("bf16", "bf16", "f32")), tokens=_log(rng, 1, 8192), width=rng.choice((64, 511, 768, 1024, 1536, 3000, 4096)),
                p=rng.choice((0.1, 0.25, 0.5)))


# --------------------------------------------------------------------------------------- states
class _State:
    """Inputs, and the buffers that a program keeps from step to step (the workspace is made by the first pass)."""

    def __init__(self, case, seed):
        self.c, self.dt, self.ws, self.lib, self.opt = case, TYPES[case["dtype"]], None, None, None
        gen = torch.Generator(device="cuda").manual_seed(int(seed))
        self._gen = gen
        _MAKE[case["op"]](self, case, int(seed))
        del self._gen

    def normal(self, *shape, std=1.0, dt=None):
        return torch.randn(*shape, device="cuda", generator=self._gen).mul_(std).to(dt or self.dt)

    def empty(self, *shape, dt=None):
        return torch.empty(*shape, dtype=dt or self.dt, device="cuda")


def _make_gated(s, c, seed):
    T, n_in, n_out, r, f32 = c["tokens"], c["n_in"], c["n_out"], c["rank"], torch.float32
    s.X = s.normal(T, n_in)
    s.V = s.normal(2 * r, n_in, std=n_in ** -0.5)
    s.U = s.normal(2, n_out, r, std=r ** -0.5)
    s.bias = s.normal(2, n_out, std=0.1, dt=f32) if c["bias"] else None
    s.H = s.dA = None
    if c["direction"] in ("infer", "forward"):
        s.A = s.empty(T, n_out)
        s.H = s.empty(T, 2 * r) if c["direction"] == "forward" else None
    else:
        s.H = (s.X.float() @ s.V.float().t()).to(s.dt)           # what the forward pass has kept
        s.dA = s.normal(T, n_out, std=1e-2)
        s.dX = s.empty(T, n_in)
        if c["direction"] == "data":
            s.dZ, s.dH = s.empty(2, T, n_out), s.empty(T, 2 * r)
        else:
            s.dV, s.dU = s.empty(2 * r, n_in, dt=f32), s.empty(2, n_out, r, dt=f32)
            s.db = s.empty(2, n_out, dt=f32) if c["bias"] else None


def _rng_state(s, seed):
    # a seed of the run and the number of the call, in device memory so that a captured step can go on counting
    s.rng = torch.tensor([(seed + 1) * SEED_MIX % 2 ** 62, 2 ** 33 + seed], dtype=torch.int64, device="cuda")


def _make_norm(s, c, seed):
    T, d, f32 = c["tokens"], c["width"], torch.float32
    rows = c["gate_rows"] or T
    stream = s.normal(T, d)
    stream[:, :: max(1, d // 5)] *= 8              # a residual stream has a few channels far larger than the others
    s.F = s.normal(T, d, std=0.7)
    s.groups = -(-T // rows)
    near_one = lambda *n: s.normal(*n, std=0.2, dt=f32).add_(1)
    s.gate = near_one(s.groups, d) if c["gate"] else None
    s.w_post = near_one(d) if c["post"] else None
    s.w_pre = near_one(d) if c["pre"] else None
    s.b_post = s.normal(d, std=0.2, dt=f32) if c["post"] and c["affine"] else None
    s.b_pre = s.normal(d, std=0.2, dt=f32) if c["pre"] and c["affine"] else None
    s.rng = None
    if c["p"]:
        _rng_state(s, seed)
    if c["direction"] == "forward":
        s.X = stream
        s.Y, s.N = s.empty(T, d), s.empty(T, d) if c["pre"] else None
    else:
        s.Y = stream                               # the stream after the block, kept by the forward pass
        s.dY, s.dN = s.normal(T, d), s.normal(T, d) if c["pre"] else None
        s.dX, s.dF = s.empty(T, d), s.empty(T, d)
        like = lambda t: None if t is None else torch.empty_like(t)
        s.dw_post, s.db_post, s.dgate, s.dw_pre, s.db_pre = (like(t) for t in (s.w_post, s.b_post, s.gate, s.w_pre, s.b_pre))


def _make_dropout(s, c, seed):
    s.X = s.normal(c["tokens"], c["width"])
    s.Y = s.empty(c["tokens"], c["width"])
    _rng_state(s, seed)


_MAKE = dict(gated=_make_gated, norm=_make_norm, dropout=_make_dropout)
EPS = 1e-5


def prepare(case, seed):
    return _State(case, seed)


# --------------------------------------------------------------------------------------- the framework's calls
def _own(s):
    c = s.c
    if s.lib is None:
        from paper_2309_03824_amd import binding
        s.lib = binding
        nbytes = 0
        if c["op"] == "gated":
            nbytes = binding.linear_gated_workspace_bytes(c["tokens"], c["n_in"], c["n_out"], c["rank"], binding.F32 if c["dtype"] == "f32" else binding.BF16, 0)
            s.act = (binding.ACT_NONE, binding.ACT_GELU, binding.ACT_SILU)[ACTS.index(c["act"])]
        if c["op"] == "norm":
            s.opt = binding.BlockNorm(kind=(binding.NORM_RMS, binding.NORM_LAYER)[NORMS.index(c["kind"])], eps=EPS, residual_scale=c["alpha"],
                                      branch_scale=c["beta"], dropout_p=c["p"], gate_rows=c["gate_rows"])
            if c["direction"] == "backward":
                nbytes = binding.block_norm_workspace_bytes(c["tokens"], c["width"])
        s.ws = torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device="cuda")
    lrd = s.lib
    if c["op"] == "dropout":
        lrd.dropout(s.X, s.Y, c["p"], s.rng)
        return dict(Y=s.Y)
    if c["op"] == "norm":
        if c["direction"] == "forward":
            lrd.block_norm_fwd(s.F, s.X, s.w_post, s.b_post, s.gate, s.w_pre, s.b_pre, s.rng, s.Y, s.N, s.opt)
            return dict(Y=s.Y, N=s.N)
        lrd.block_norm_bwd(s.dY, s.dN, s.F, s.Y, s.w_post, s.b_post, s.gate, s.w_pre, s.rng, s.dX, s.dF, s.dw_post, s.db_post, s.dgate, s.dw_pre, s.db_pre,
                           s.opt, s.ws)
        return dict(dX=s.dX, dF=s.dF, dw_post=s.dw_post, db_post=s.db_post, dgate=s.dgate, dw_pre=s.dw_pre, db_pre=s.db_pre)
    if c["direction"] in ("infer", "forward"):
        lrd.linear_gated_fwd(s.X, s.V, s.U, s.bias, s.A, s.H, s.act, s.ws)
        return dict(A=s.A, H=s.H)
    if c["direction"] == "data":
        lrd.linear_gated_bwd_data(s.dA, s.H, s.V, s.U, s.bias, s.dX, s.dZ, s.dH, s.act, s.ws)
        return dict(dX=s.dX, dZ=s.dZ, dH=s.dH)
    lrd.linear_gated_bwd(s.dA, s.X, s.H, s.V, s.U, s.bias, s.dX, s.dV, s.dU, s.db, 0, s.act, s.ws)
    return _exchanged(dict(dX=s.dX, dV=s.dV, dU=s.dU, db=s.db), s.dt)


def _exchanged(out, dt):
    """The gradients as data-parallel ranks exchange them, in the type of the weights."""
    return {k: None if v is None else v.to(dt) for k, v in out.items()}


# --------------------------------------------------------------------------------------- the plain form
def _act(z, name):
    """act(z) and its derivative."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "silu":
        p = 1 / (1 + torch.exp(-z))
        return z * p, p * (1 + z * (1 - p))
    cdf = 0.5 * (1 + torch.erf(z * 2 ** -0.5))
    return z * cdf, cdf + z * torch.exp(-0.5 * z * z) * (2 * torch.pi) ** -0.5


def _plain_gated(s):
    c, r = s.c, s.c["rank"]
    V, U = s.V.float(), s.U.float()
    bg, bu = s.bias if s.bias is not None else (0.0, 0.0)
    infer = c["direction"] in ("infer", "forward")
    stored = (s.X.float() @ V.t()).to(s.dt) if infer else s.H
    Hg, Hu = stored[:, :r].float(), stored[:, r:].float()
    zg, zu = Hg @ U[0].t() + bg, Hu @ U[1].t() + bu
    a, da = _act(zg, c["act"])
    if infer:
        return dict(A=(a * zu).to(s.dt), H=stored if c["direction"] == "forward" else None)
    dA = s.dA.float()
    dZ = torch.stack((dA * zu * da, dA * a)).to(s.dt)
    g, u = dZ[0].float(), dZ[1].float()
    dH = torch.cat((g @ U[0], u @ U[1]), 1).to(s.dt)
    dX = (dH.float() @ V).to(s.dt)
    if c["direction"] == "data":
        return dict(dX=dX, dZ=dZ, dH=dH)
    dV, dU = dH.float().t() @ s.X.float(), torch.stack((g.t() @ Hg, u.t() @ Hu))
    return _exchanged(dict(dX=dX, dV=dV, dU=dU, db=torch.stack((g.sum(0), u.sum(0))) if s.bias is not None else None), s.dt)


def _bits16(rng, n):
    """16 random bits for each of n elements: Philox4x32 with 10 rounds (Salmon, Moraes, Dror, Shaw 2011), key = the seed, counter =
    (element / 8, the call's number), the eight 16-bit halves of its four words in order."""
    low = 0xFFFFFFFF
    group = torch.arange((n + 7) // 8, dtype=torch.int64, device=rng.device)
    k0, k1 = rng[0] & low, (rng[0] >> 32) & low
    c = [group & low, group >> 32, (rng[1] & low).expand_as(group), ((rng[1] >> 32) & low).expand_as(group)]
    for _ in range(10):          # the generator's rounds
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((b >> 32) & low) ^ c[1] ^ k0, b & low, ((a >> 32) & low) ^ c[3] ^ k1, a & low]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    w = torch.stack(c, 1)
    return torch.stack((w & 0xFFFF, w >> 16), 2).reshape(-1)[:n]


def _keep(rng, p, shape):
    """The elements that stay, and their scale: an element is dropped where its 16 bits are below p 65536."""
    below = round(p * 65536)
    n = shape[0] * shape[1]
    return (_bits16(rng, n) >= below).reshape(shape), 65536 / (65536 - below)


def _plain_dropout(s):
    keep, scale = _keep(s.rng, s.c["p"], s.X.shape)
    return dict(Y=torch.where(keep, s.X.float() * scale, 0.0).to(s.dt))


def _norm(x, kind):
    """The normalised rows and 1 / their root."""
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    inv = 1 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)
    return x * inv, inv


def _norm_grad(g, xhat, inv, kind):
    """The gradient of the rows from that of the normalised ones."""
    d = g - xhat * (g * xhat).mean(1, keepdim=True)
    return inv * (d - g.mean(1, keepdim=True) if kind == "layer" else d)


def _plain_norm(s):
    c, kind = s.c, s.c["kind"]
    T, d, rows = c["tokens"], c["width"], c["gate_rows"] or c["tokens"]
    gate = s.gate.repeat_interleave(rows, 0)[:T] if s.gate is not None else None
    times = lambda a, b: a if b is None else a * b
    plus = lambda a, b: a if b is None else a + b
    F = s.F.float()
    z = F
    if c["post"]:
        fhat, finv = _norm(F, kind)
        z = plus(fhat * s.w_post, s.b_post)
    keep, scale = _keep(s.rng, c["p"], F.shape) if c["p"] else (None, 1.0)
    drop = (lambda t: torch.where(keep, t * scale, 0.0)) if c["p"] else lambda t: t
    if c["direction"] == "forward":
        y = c["alpha"] * s.X.float() + c["beta"] * drop(times(z, gate))
        n = plus(_norm(y, kind)[0] * s.w_pre, s.b_pre).to(s.dt) if c["pre"] else None
        return dict(Y=y.to(s.dt), N=n)
    g, out = s.dY.float(), dict(dw_post=None, db_post=None, dgate=None, dw_pre=None, db_pre=None)
    if c["pre"]:
        dN = s.dN.float()
        yhat, yinv = _norm(s.Y.float(), kind)
        g = g + _norm_grad(dN * s.w_pre, yhat, yinv, kind)
        out["dw_pre"] = (dN * yhat).sum(0)
        out["db_pre"] = dN.sum(0) if s.b_pre is not None else None
    e = c["beta"] * drop(g)
    if s.gate is not None:
        short = s.groups * rows - T
        out["dgate"] = torch.cat((e * z, e.new_zeros(short, d))).reshape(s.groups, rows, d).sum(1)
    dz = times(e, gate)
    dF = dz
    if c["post"]:
        out["dw_post"] = (dz * fhat).sum(0)
        out["db_post"] = dz.sum(0) if s.b_post is not None else None
        dF = _norm_grad(dz * s.w_post, fhat, finv, kind)
    return dict(out, dX=(c["alpha"] * g).to(s.dt), dF=dF.to(s.dt))


_PLAIN = dict(gated=_plain_gated, norm=_plain_norm, dropout=_plain_dropout)


def run(state):
    if own:
        return _own(state)
    return _PLAIN[state.c["op"]](state)


# --------------------------------------------------------------------------------------- the definitions in 64 bits
def _exact_act(z, name):
    if name == "none":
        return z, 1.0
    if name == "silu":
        e = torch.sigmoid(z)
        return z * e, e + z * e * torch.sigmoid(-z)
    phi = torch.special.ndtr(z)
    return z * phi, phi + z * torch.exp(-z * z / 2) / (2 * np.pi) ** 0.5


def _exact_gated(s):
    c, r, dt = s.c, s.c["rank"], s.dt
    Vg, Vu, Ug, Uu = (t.double() for t in (s.V[:r], s.V[r:], s.U[0], s.U[1]))
    X = s.X.double()
    kept = lambda t: t.to(dt).double()               # an intermediate in the type of the activations
    if c["direction"] in ("infer", "forward"):
        whole_hg, whole_hu = X @ Vg.mT, X @ Vu.mT
        hg, hu = kept(whole_hg), kept(whole_hu)
    else:
        hg, hu = s.H[:, :r].double(), s.H[:, r:].double()
    zg, zu = hg @ Ug.mT, hu @ Uu.mT
    if s.bias is not None:
        zg, zu = zg + s.bias[0].double(), zu + s.bias[1].double()
    a, slope = _exact_act(zg, c["act"])
    if c["direction"] in ("infer", "forward"):
        return dict(A=a * zu, H=torch.hstack((whole_hg, whole_hu)) if c["direction"] == "forward" else None)
    dA = s.dA.double()
    whole_g, whole_u = dA * zu * slope, dA * a
    dzg, dzu = kept(whole_g), kept(whole_u)
    whole_hg, whole_hu = dzg @ Ug, dzu @ Uu
    dhg, dhu = kept(whole_hg), kept(whole_hu)
    dX = dhg @ Vg + dhu @ Vu
    if c["direction"] == "data":
        return dict(dX=dX, dZ=torch.stack((whole_g, whole_u)), dH=torch.hstack((whole_hg, whole_hu)))
    db = torch.stack((dzg.sum(0), dzu.sum(0))) if s.bias is not None else None
    return dict(dX=dX, dV=torch.vstack((dhg.mT @ X, dhu.mT @ X)), dU=torch.stack((dzg.mT @ hg, dzu.mT @ hu)), db=db)


def _exact_mask(s, T, d, p):
    """What each element is multiplied by, from the generator in unsigned integers on the host."""
    seed, call = (int(v) & (2 ** 64 - 1) for v in s.rng.tolist())
    n, low, half = T * d, np.uint64(0xFFFFFFFF), np.uint64(32)
    at = np.arange(-(-n // 8), dtype=np.uint64)
    x0, x1 = at & low, at >> half
    x2, x3 = np.full_like(at, call & 0xFFFFFFFF), np.full_like(at, call >> 32)
    for i in range(10):
        key0, key1 = np.uint64((seed + i * 0x9E3779B9) & 0xFFFFFFFF), np.uint64(((seed >> 32) + i * 0xBB67AE85) & 0xFFFFFFFF)
        p0, p1 = x0 * np.uint64(0xD2511F53), x2 * np.uint64(0xCD9E8D57)
        x0, x1, x2, x3 = (p1 >> half) ^ x1 ^ key0, p1 & low, (p0 >> half) ^ x3 ^ key1, p0 & low
    words = np.stack((x0, x1, x2, x3), axis=1).astype("<u4")
    bits = words.view("<u2").reshape(-1)[:n]
    below = int(np.rint(p * 65536))
    return torch.from_numpy((bits >= below) * (65536.0 / (65536 - below))).reshape(T, d).to(s.rng.device)


def _exact_dropout(s):
    return dict(Y=s.X.double() * _exact_mask(s, s.c["tokens"], s.c["width"], s.c["p"]))


def _exact_norm(s):
    c, layer = s.c, s.c["kind"] == "layer"
    T, d = c["tokens"], c["width"]
    of = torch.arange(T, device="cuda") // (c["gate_rows"] or T)
    gate = s.gate.double()[of] if s.gate is not None else 1.0
    factor = c["beta"] * (_exact_mask(s, T, d, c["p"]) if c["p"] else 1.0)
    opt = lambda t, other: other if t is None else t.double()

    def unit(x):
        centred = x - x.sum(1, keepdim=True) / d if layer else x
        std = (centred.square().sum(1, keepdim=True) / d + EPS).sqrt()
        return centred / std, std

    def back(g, hat, std):
        g = g - hat * (g * hat).sum(1, keepdim=True) / d - (g.sum(1, keepdim=True) / d if layer else 0.0)
        return g / std

    F = s.F.double()
    fhat, fstd = unit(F)
    z = fhat * s.w_post.double() + opt(s.b_post, 0.0) if c["post"] else F
    if c["direction"] == "forward":
        y = c["alpha"] * s.X.double() + factor * gate * z
        return dict(Y=y, N=unit(y)[0] * s.w_pre.double() + opt(s.b_pre, 0.0) if c["pre"] else None)
    total, grads = s.dY.double(), {}
    if c["pre"]:
        dN = s.dN.double()
        hat, std = unit(s.Y.double())
        total = total + back(dN * s.w_pre.double(), hat, std)
        grads["dw_pre"] = (dN * hat).sum(0)
        grads["db_pre"] = dN.sum(0) if s.b_pre is not None else None
    inner = total * factor
    if s.gate is not None:
        grads["dgate"] = torch.zeros(s.groups, d, dtype=torch.float64, device="cuda").index_add_(0, of, inner * z)
    dz = inner * gate
    if c["post"]:
        grads["dw_post"] = (dz * fhat).sum(0)
        grads["db_post"] = dz.sum(0) if s.b_post is not None else None
    return dict(grads, dX=c["alpha"] * total, dF=back(dz * s.w_post.double(), fhat, fstd) if c["post"] else dz)


_EXACT = dict(gated=_exact_gated, norm=_exact_norm, dropout=_exact_dropout)


def exact(case, seed):
    return _EXACT[case["op"]](prepare(case, seed))


# --------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    c, e = case, 2 if case["dtype"] == "bf16" else 4
    T = c["tokens"]
    if c["op"] == "dropout":
        return {"bytes": 2 * e * T * c["width"], "flops": 0}
    if c["op"] == "norm":
        d, back = c["width"], c["direction"] == "backward"
        groups = -(-T // (c["gate_rows"] or T)) if c["gate"] else 0
        params = (c["post"] + c["pre"]) * (1 + c["affine"]) + groups
        # forward F, X -> Y, N; backward dY, dN, Y (for the norm before) and F (for the norm behind, or the gate) -> dX, dF
        big = 3 + c["pre"] if not back else 3 + 2 * c["pre"] + (c["post"] or c["gate"])
        return {"bytes": e * T * d * big + 4 * d * params * (1 + back), "flops": 0}
    n_in, n_out, r = c["n_in"], c["n_out"], c["rank"]
    weights, pair = e * 2 * r * (n_in + n_out) + (8 * n_out if c["bias"] else 0), 4 * T * r
    if c["direction"] in ("infer", "forward"):
        return {"bytes": weights + e * T * (n_in + n_out + (2 * r if c["direction"] == "forward" else 0)), "flops": pair * (n_in + n_out)}
    nbytes, flops = weights + e * T * (n_out + 2 * r + n_in), pair * (2 * n_out + n_in)
    if c["direction"] == "data":
        return {"bytes": nbytes + e * T * (2 * n_out + 2 * r), "flops": flops}
    return {"bytes": nbytes + e * T * n_in + 8 * r * (n_in + n_out) + (8 * n_out if c["bias"] else 0), "flops": flops + pair * (n_in + n_out)}
