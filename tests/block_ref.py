"""The operators between and around the decomposed layers of a feed-forward block, plainly in 64 bits, and how far fp32 arithmetic may
take a result from them.

U = 2^-24 is half a step of fp32 (relative).  A sum of n terms in fp32, in any order, is off by at most n U sum|terms| (first
order); bounds below are such first-order sums, doubled by SAFE for the second-order rest."""
import numpy as np
import torch

U = 2.0 ** -24
SAFE = 2.0
ACTS = {0: "none", 1: "gelu", 2: "silu"}


def half_step(dt):
    return torch.finfo(dt).eps / 2


# ------------------------------------------------------------------------------------------ dropout
def philox4x32(ctr, key, rounds=10):
    """Words [n, 4] for counters [n, 4] and a key of two words, in unsigned 64-bit integers (Salmon, Moraes, Dror, Shaw 2011)."""
    c = [np.asarray(ctr)[:, i].astype(np.uint64) for i in range(4)]
    k, low, half = [int(key[0]), int(key[1])], np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> half) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> half) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, 1).astype(np.uint32)


def drop_factors(n, p, seed, call, first=0):
    """What elements first .. first + n - 1 are multiplied by: 0 or the scale, rounded to fp32 as the library has it (64-bit tensor)."""
    seed, call = seed % 2 ** 64, call % 2 ** 64
    g0 = first // 8
    g = np.arange(g0, (first + n + 7) // 8, dtype=np.uint64)
    ctr = np.stack((g & np.uint64(0xFFFFFFFF), g >> np.uint64(32), np.full_like(g, call & 0xFFFFFFFF), np.full_like(g, call >> 32)), 1)
    words = philox4x32(ctr, (seed & 0xFFFFFFFF, seed >> 32))
    bits = np.stack((words & 0xFFFF, words >> 16), 2).reshape(-1)[first - 8 * g0:][:n]
    below = round(p * 65536)
    scale = float(np.float32(65536 / (65536 - below))) if below < 65536 else 0.0
    return torch.from_numpy(np.where(bits >= below, scale, 0.0))


# ------------------------------------------------------------------------------------------ gated pair
def act_terms(z, act):
    """act(z), act'(z)."""
    if act == 0:
        return z, torch.ones_like(z)
    if act == 2:
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    phi = torch.exp(-z * z / 2) / (2 * np.pi) ** 0.5
    cdf = torch.special.ndtr(z)
    return z * cdf, cdf + z * phi


def act_errors(z, act, dt):
    """How far the library's act(z), act'(z) may be off at the fp32 value z.
    GELU in bf16: the polynomials' 1.2e-4 of Phi and 2.6e-4 of the derivative.  In fp32: Phi by a rational form of 7.5e-8, in whose
    evaluation five steps of coefficients below 1.5, a reciprocal and an exponential (relative (z^2 / 2 + 2) 2^-23) add under 1e-6, and
    1.5e-6 to the derivative.  SiLU: s = 1 / (1 + e), e = exp(-z) relative (1.5 |z| + 2) 2^-24 off by the rounded
    exponent and the instruction, of which 1 - s reaches s, and a reciprocal of one step: s off by s ((1 - s)(1.5 |z| + 2) + 4) U."""
    if act == 0:
        return torch.zeros_like(z), torch.zeros_like(z)
    if act == 1:
        p, d = (1.2e-4, 2.6e-4) if dt == torch.bfloat16 else (1e-6, 1.5e-6)
        return p * z.abs() + 4 * U * z.abs(), torch.full_like(z, d)
    s = torch.sigmoid(z)
    es = s * ((1 - s) * (1.5 * z.abs() + 2) + 4) * U
    return z.abs() * (es + 2 * U * s), es * (1 + 2 * z.abs()) + 6 * U * (1 + z.abs()) * s


def product(a, b, terms=0):
    """a @ b.T in 64 bits, and the bound of its fp32 sum of K products (+ `terms` more roundings)."""
    c = a @ b.t()
    return c, (a.shape[1] + 2 + terms) * U * (a.abs() @ b.abs().t())


def gated(H, Uc, bias, act, dt, dA=None):
    """From the stored H [T, 2r]: (A, its bound), or with dA ((dZg, bound), (dZu, bound)); before the last rounding."""
    r = Uc.shape[2]
    zs = []
    for k in range(2):
        z, e = product(H[:, k * r:(k + 1) * r], Uc[k])
        if bias is not None:
            z = z + bias[k]
            e = e + U * (z.abs() + bias[k].abs())
        zs.append((z, e))
    (zg, eg), (zu, eu) = zs
    a, da = act_terms(zg, act)
    ea, eda = act_errors(zg, act, dt if dA is None else torch.float32)       # (backward in fp32's accuracy whatever the type)
    ea, eda = ea + 1.13 * eg, eda + 0.8 * eg                  # |act'| <= 1.13, |act''| <= 0.8
    if dA is None:
        return a * zu, SAFE * (zu.abs() * ea + a.abs() * eu + ea * eu + 2 * U * (a * zu).abs())
    d = dA.abs()
    g, u = dA * zu * da, dA * a
    return ((g, SAFE * (d * (zu.abs() * eda + da.abs() * eu + eda * eu) + 3 * U * g.abs())), (u, SAFE * (d * ea + 2 * U * u.abs())))


# ------------------------------------------------------------------------------------------ block norm
SUM = 64          # roundings that a sum over a row goes through: 16 columns of a thread, 6 levels of a wave, 16 waves, and what enters it


def normalise(x, ex, layer, eps):
    """(normalised rows, bound, 1 / root, its relative bound) of x, which is off by at most ex."""
    mean = lambda t: t.mean(1, keepdim=True)
    m = mean(x) if layer else 0.0
    c = x - m
    ec = ex + U * c.abs() + (mean(ex) + SUM * U * mean(x.abs()) if layer else 0.0)
    inv = 1 / torch.sqrt(mean(c * c) + eps)
    rel = inv * inv * (mean(c.abs() * ec) + mean(ec * ec)) + SUM * U
    hat = c * inv
    return hat, inv * ec + hat.abs() * rel + ec * inv * rel, inv, rel


def normalise_grad(g, eg, hat, ehat, inv, rel, layer):
    mean = lambda t: t.mean(1, keepdim=True)
    along, m = mean(g * hat), mean(g) if layer else 0.0
    ealong = mean(eg * hat.abs() + g.abs() * ehat) + SUM * U * mean((g * hat).abs())
    em = mean(eg) + SUM * U * mean(g.abs()) if layer else 0.0
    d = inv * (g - m - hat * along)
    size = g.abs() + (m.abs() if layer else 0.0) + (hat * along).abs()
    return d, inv * (eg + em + hat.abs() * ealong + ehat * along.abs() + 4 * U * size) + rel * inv * size


def block_norm_fwd(F, X, w_post, b_post, gate, w_pre, b_pre, factors, o):
    """Y and N before their last rounding, with bounds: ((Y, eY), (N, eN)); o: dict(layer, eps, alpha, beta, gate_rows)."""
    T = X.shape[0]
    if F is None:
        y, ey = X, torch.zeros_like(X)
    else:
        z, ez = F, torch.zeros_like(F)
        if w_post is not None:
            hat, eh, _, _ = normalise(F, ez, o["layer"], o["eps"])
            z = hat * w_post + (0.0 if b_post is None else b_post)
            ez = eh * w_post.abs() + 2 * U * ((hat * w_post).abs() + z.abs())
        if gate is not None:
            row = gate[torch.arange(T) // (o["gate_rows"] or T)]
            z, ez = z * row, ez * row.abs() + U * (z * row).abs()
        if factors is not None:
            z, ez = z * factors, ez * factors + U * (z * factors).abs()
        y = o["alpha"] * X + o["beta"] * z
        ey = abs(o["beta"]) * ez + 3 * U * (abs(o["alpha"]) * X.abs() + abs(o["beta"]) * z.abs())
    if w_pre is None:
        return (y, SAFE * ey), None
    hat, eh, _, _ = normalise(y, ey, o["layer"], o["eps"])
    n = hat * w_pre + (0.0 if b_pre is None else b_pre)
    return (y, SAFE * ey), (n, SAFE * (eh * w_pre.abs() + 2 * U * ((hat * w_pre).abs() + n.abs())))


def block_norm_bwd(dY, dN, F, Y, w_post, b_post, gate, w_pre, factors, o):
    """dict of (gradient, bound), before the last rounding."""
    like = dY if dY is not None else dN
    T, d = like.shape
    out = {}
    add = T + 600                 # roundings of a sum over tokens: rows of a thread, slots, and the partial rows

    def tokens(t, et):
        return t.sum(0), SAFE * (et.sum(0) + add * U * t.abs().sum(0))

    up, eup = (dY, torch.zeros_like(dY)) if dY is not None else (torch.zeros_like(dN), torch.zeros_like(dN))
    if dN is not None:
        hat, eh, inv, rel = normalise(Y, torch.zeros_like(Y), o["layer"], o["eps"])
        out["dw_pre"] = tokens(dN * hat, dN.abs() * eh)
        out["db_pre"] = tokens(dN, torch.zeros_like(dN))
        g = dN * w_pre
        g, eg = normalise_grad(g, U * g.abs(), hat, eh, inv, rel, o["layer"])
        up, eup = up + g, eg + U * (up + g).abs()
    out["dX"] = o["alpha"] * up, SAFE * (abs(o["alpha"]) * (eup + U * up.abs()))
    if F is None and (w_post is not None):
        return out
    e, ee = o["beta"] * up, abs(o["beta"]) * (eup + U * up.abs())
    if factors is not None:
        e, ee = e * factors, factors * (ee + U * e.abs())
    z, ez = F, None
    if F is not None:
        z, ez = F, torch.zeros_like(F)
        if w_post is not None:
            hat, eh, inv, rel = normalise(F, ez, o["layer"], o["eps"])
            z = hat * w_post + (0.0 if b_post is None else b_post)
            ez = eh * w_post.abs() + 2 * U * ((hat * w_post).abs() + z.abs())
    if gate is not None:
        rows = o["gate_rows"] or T
        if z is not None:
            t, et = e * z, ee * z.abs() + e.abs() * ez
            of = torch.arange(T) // rows
            zero = torch.zeros(gate.shape, dtype=torch.float64)
            out["dgate"] = zero.index_add(0, of, t), SAFE * (zero.index_add(0, of, et) + add * U * zero.index_add(0, of, t.abs()))
        row = gate[torch.arange(T) // rows]
        e, ee = e * row, row.abs() * (ee + U * e.abs())
    if w_post is not None:
        out["dw_post"] = tokens(e * hat, ee * hat.abs() + e.abs() * eh)
        out["db_post"] = tokens(e, ee)
        g = e * w_post
        e, ee = normalise_grad(g, ee * w_post.abs() + U * g.abs(), hat, eh, inv, rel, o["layer"])
    out["dF"] = e, SAFE * ee
    return out


def assert_close(got, want, dt, what):
    """got (a device tensor of type dt) against (value, bound before the last rounding)."""
    value, err = want
    got = got.detach().cpu()
    assert got.dtype == dt and got.shape == value.shape, (what, got.dtype, got.shape, value.shape)
    got = got.double()
    assert torch.isfinite(got).all(), what
    allowed = err + half_step(dt) * (value.abs() + err) + torch.finfo(torch.float32).tiny
    off = (got - value).abs() - allowed
    worst = int(off.argmax())
    assert off.max() <= 0, (what, "off by", float((got - value).abs().flatten()[worst]), "allowed", float(allowed.flatten()[worst]), "at", worst,
                            "value", float(value.flatten()[worst]))
