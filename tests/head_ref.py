"""The head operators in 64 bits, from their definitions (plain torch on whatever device the inputs are on)."""
import math

import torch

U32 = 2.0 ** -24                 # half a step of fp32, relative


def act(name, z):
    if name == "relu":
        return z.clamp_min(0)
    if name == "leaky":
        return torch.where(z > 0, z, 0.1 * z)
    if name == "sigmoid":
        return torch.sigmoid(z)
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return z * 0.5 * (1 + torch.erf(z / math.sqrt(2)))
    return z


def norm(x, groups, gamma, beta, eps, name):
    """(y, mean, rstd) of x [n, ..., c] in float64."""
    n, c = x.shape[0], x.shape[-1]
    v = x.double().reshape(n, -1, groups, c // groups)
    mean = v.mean(dim=(1, 3), keepdim=True)
    rstd = ((v - mean).square().mean(dim=(1, 3), keepdim=True) + eps).rsqrt()
    z = ((v - mean) * rstd).reshape(n, -1, c)
    if gamma is not None:
        z = z * gamma.double()
    if beta is not None:
        z = z + beta.double()
    return act(name, z).reshape(x.shape), mean.reshape(n, groups), rstd.reshape(n, groups)


def scan(g, x, h0, reset=None, lengths=None):
    """(h, last) in float64; rows of h behind a stream's last frame are zero."""
    T, n, d = g.shape
    f = torch.sigmoid(g.double())
    take = torch.sigmoid(-g.double())
    s = torch.zeros(n, d, dtype=torch.float64, device=g.device) if h0 is None else h0.double()
    out = []
    for t in range(T):
        before = s if reset is None else torch.where(reset[t].bool()[:, None], torch.zeros_like(s), s)
        h = f[t] * before + take[t] * x[t].double()
        on = torch.ones(n, 1, dtype=torch.bool, device=g.device) if lengths is None else (t < lengths)[:, None]
        s = torch.where(on, h, s)
        out.append(torch.where(on, h, torch.zeros_like(h)))
    return (torch.stack(out) if out else torch.zeros(0, n, d, dtype=torch.float64, device=g.device)), s


def gated_ff(x, wg, wu, bg, bu, name):
    x, wg, wu = x.double(), wg.double(), wu.double()
    g, u = x @ wg.t(), x @ wu.t()
    if bg is not None:
        g = g + bg.double()
    if bu is not None:
        u = u + bu.double()
    return act(name, g) * u


def close(got, want, tol, what=""):
    """Elementwise |got - want| <= tol (a tensor or a number), NaNs nowhere."""
    err = (got.double() - want).abs()
    tol = torch.as_tensor(tol, dtype=torch.float64, device=err.device).expand_as(err)
    bad = ~(err <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err - tol).max()):.3g} over, error {float(err.max()):.3g}"


def half_step(t, like):
    """Half a step of type t at the values `like`, and the smallest step below the normal numbers."""
    i = torch.finfo(t)
    return i.eps / 2 * like.abs() + i.smallest_normal * i.eps / 2
