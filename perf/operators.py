"""Cases of the operators that a recurrent head on a video network's feature maps is made of: group normalisation with an
activation (channels last), the gated feed-forward block and the gated linear recurrence over frames, each forward and backward.

`run` evaluates a case in plain elementary operations, or with `own` set through the library's entry points; `exact` gives the
same outputs from the definitions in 64 bits."""
import math

import torch

own = False

_T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5


def listed():
    return [
        # one frame's 56x56x64 feature map of a lone fp32 convolution, normalised as it arrives: launch latency counts
        dict(name="norm f32 one frame", op="norm", dtype="f32", n=1, h=56, w=56, c=64, groups=32, act="relu", pad=0),
        # a chunk of 32 AlexNet-shaped frames after the second convolution's pool
        dict(name="norm bf16 chunk", op="norm", dtype="bf16", n=32, h=27, w=27, c=256, groups=32, act="silu", pad=0),
        # a training batch of 64 ResNet-18-shaped frames at the first layer's 112x112 resolution
        dict(name="norm backward bf16 batch", op="norm_backward", dtype="bf16", n=64, h=112, w=112, c=64, groups=32, act="silu", pad=0),
        # few odd feature maps, 12 channels a group, read as a slice of wider rows
        dict(name="norm backward f16 ragged", op="norm_backward", dtype="f16", n=3, h=13, w=17, c=84, groups=7, act="gelu", pad=4),
        # one frame of one video through a block of fc6's shape: the weights have to be streamed once
        dict(name="ff bf16 one frame", op="ff", dtype="bf16", m=1, k=9216, f=4096, act="silu", bias=True, pad=0),
        # 64 frames of 32 videos at once: the largest call
        dict(name="ff bf16 chunk", op="ff", dtype="bf16", m=2048, k=9216, f=4096, act="silu", bias=False, pad=0),
        # fp32 features of an odd number of frames into as many gates as there are classes, and one
        dict(name="ff f32 ragged", op="ff", dtype="f32", m=77, k=1000, f=1001, act="gelu", bias=True, pad=3),
        # a training step of the block on 1024 frames
        dict(name="ff backward bf16", op="ff_backward", dtype="bf16", m=1024, k=4096, f=4096, act="silu", bias=True, pad=0),
        # one frame of four videos: the serving step
        dict(name="scan f32 one frame", op="scan", dtype="f32", t=1, n=4, d=4096, resets=True, lengths=False, packed=True),
        # two long videos whose features are pooled to ResNet-18's 512, with scene cuts
        dict(name="scan bf16 long", op="scan", dtype="bf16", t=16384, n=2, d=512, resets=True, lengths=False, packed=True),
        # a training batch of clips of unequal lengths, padded to the longest
        dict(name="scan backward bf16 batch", op="scan_backward", dtype="bf16", t=512, n=32, d=1024, resets=False, lengths=True, packed=False),
        # few fp32 clips, odd in every size
        dict(name="scan backward f32 ragged", op="scan_backward", dtype="f32", t=1023, n=3, d=333, resets=True, lengths=True, packed=False),
    ]


def _log(rng, lo, hi):
    """A whole number whose logarithm is spread evenly over [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm_backward", "ff", "ff_backward", "scan", "scan_backward"])
    if op in ("norm", "norm_backward"):
        dtype = rng.choice(["f32", "bf16", "f16"])
        while True:
            groups = rng.choice([1, 2, 3, 4, 7, 8, 16, 32, 32])
            c = groups * _log(rng, 1, 64)
            n, h, w = _log(rng, 1, 64), _log(rng, 1, 112), _log(rng, 1, 112)
            if c <= 512 and n * h * w * c <= 24_000_000 and h * w * c >= 16 * groups:   # a group of few values leaves no gradient
                break
        act = rng.choice(["none", "relu", "leaky", "silu", "gelu"] if op == "norm" else ["none", "silu", "gelu"])
        return dict(op=op, dtype=dtype, n=n, h=h, w=w, c=c, groups=groups, act=act, pad=rng.choice([0, 0, 1, 8]))
    if op in ("ff", "ff_backward"):
        dtype = rng.choice(["f32", "bf16"])
        most = 1024 if op == "ff_backward" else 2048
        m, k, f = _log(rng, 1, most), _log(rng, 16, 9216 if op == "ff" else 4096), _log(rng, 16, 4096)
        if rng.random() < 0.5:
            k, f = max(16, k // 64 * 64), max(16, f // 64 * 64)
        return dict(op=op, dtype=dtype, m=m, k=k, f=f, act=rng.choice(["none", "sigmoid", "silu", "gelu"]), bias=rng.random() < 0.5,
                    pad=rng.choice([0, 0, 1, 8]))
    dtype = rng.choice(["f32", "bf16", "f16"])
    while True:
        t, n, d = _log(rng, 1, 16384), _log(rng, 1, 32), _log(rng, 1, 4096)
        if t * n * d <= 16_000_000:
            break
    return dict(op=op, dtype=dtype, t=t, n=n, d=d, resets=rng.random() < 0.5, lengths=rng.random() < 0.5, packed=rng.random() < 0.5)


def _lengths(c):
    """Frames of each stream: the first has all of them, the last little more than half."""
    return [c["t"] - (i * c["t"]) // (2 * c["n"]) for i in range(c["n"])]


def prepare(case, seed):
    c = dict(case)
    r = torch.Generator(device="cuda")
    r.manual_seed(seed)
    dt = _T[c["dtype"]]

    def normal(*shape, scale=1.0, to=dt):
        return (torch.randn(*shape, generator=r, device="cuda") * scale).to(to)

    def rows(last, *shape, scale=1.0):
        """Rows of `last` values, `pad` apart: a slice of a wider buffer."""
        return normal(*shape, last + c["pad"], scale=scale)[..., :last]

    s = {"case": c}
    if c["op"].startswith("norm"):
        n, h, w, ch, g = c["n"], c["h"], c["w"], c["c"], c["groups"]
        # projections: each channel has a mean and a spread of its own
        x = torch.randn(n, h, w, ch + c["pad"], generator=r, device="cuda")
        x = x * (0.5 + torch.rand(ch + c["pad"], generator=r, device="cuda")) + torch.randn(ch + c["pad"], generator=r, device="cuda")
        s["x"] = x.to(dt)[..., :ch]
        s["gamma"] = 1 + normal(ch, scale=0.2, to=torch.float32)
        s["beta"] = normal(ch, scale=0.2, to=torch.float32)
        if c["op"] == "norm_backward":
            s["dy"] = normal(n, h, w, ch)
            v = s["x"].double().reshape(n, h * w, g, ch // g)
            var, mean = torch.var_mean(v, dim=(1, 3), correction=0)
            s["stats"] = torch.stack([mean, (var + EPS).rsqrt()], -1).float().contiguous()   # as the forward pass left them
    elif c["op"].startswith("ff"):
        m, k, f = c["m"], c["k"], c["f"]
        s["x"] = rows(k, m)
        s["wg"], s["wu"] = rows(k, f, scale=k ** -0.5), rows(k, f, scale=k ** -0.5)
        s["bg"] = normal(f, scale=0.1, to=torch.float32) if c["bias"] else None
        s["bu"] = normal(f, scale=0.1, to=torch.float32) if c["bias"] else None
        if c["op"] == "ff_backward":
            s["dy"] = normal(m, f)
    else:
        t, n, d = c["t"], c["n"], c["d"]
        if c["packed"]:   # gates and values are the halves of one projection's rows
            both = normal(t, n, 2 * d)
            both[..., :d] += 2
            s["g"], s["x"] = both[..., :d], both[..., d:]
        else:
            s["g"], s["x"] = normal(t, n, d) + 2, normal(t, n, d)
        s["h0"] = normal(n, d, to=torch.float32)
        s["reset"] = (torch.rand(t, n, generator=r, device="cuda") < 0.02).to(torch.uint8) if c["resets"] else None
        s["lengths"] = torch.tensor(_lengths(c), dtype=torch.int32, device="cuda") if c["lengths"] else None
        if c["op"] == "scan_backward":
            s["dh"] = normal(t, n, d)
            s["dlast"] = normal(n, d, to=torch.float32)
    return s


# ---- the calls a user makes ----------------------------------------------------------------------------------------

def _own(s):
    import paper_1802_09723_b200 as rrm

    c = s["case"]
    op = c["op"]
    if op == "norm":
        return rrm.group_norm(s["x"], c["groups"], s["gamma"], s["beta"], eps=EPS, act=c["act"])
    if op == "norm_backward":
        return rrm.group_norm_backward(s["x"], s["dy"], c["groups"], s["gamma"], s["beta"], s["stats"], act=c["act"])
    if op == "ff":
        return rrm.gated_ff(s["x"], s["wg"], s["wu"], s["bg"], s["bu"], act=c["act"])
    if op == "ff_backward":
        return rrm.gated_ff_backward(s["x"], s["wg"], s["wu"], s["dy"], s["bg"], s["bu"], act=c["act"])
    if op == "scan":
        return rrm.gated_scan(s["g"], s["x"], s["h0"], reset=s["reset"], lengths=s["lengths"])
    return rrm.gated_scan_backward(s["g"], s["x"], s["dh"], s["h0"], s["dlast"], reset=s["reset"], lengths=s["lengths"])


# ---- the plain form ------------------------------------------------------------------------------------------------

def _normal_cdf(z):
    return 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))


def _act(name, z):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "leaky":
        return torch.where(z > 0, z, 0.1 * z)
    if name == "sigmoid":
        return 1 / (1 + torch.exp(-z))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "gelu":
        return z * _normal_cdf(z)
    return z


def _slope(name, z):
    if name in ("sigmoid", "silu"):
        q = 1 / (1 + torch.exp(-z))
        return q * (1 - q) if name == "sigmoid" else q * (1 + z * (1 - q))
    if name == "gelu":
        return _normal_cdf(z) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    return torch.ones_like(z)


def _norm(s):
    c, x = s["case"], s["x"]
    shape = (c["n"], c["h"] * c["w"], c["groups"], c["c"] // c["groups"])
    v = x.float().reshape(shape)
    mean = v.mean(dim=(1, 3), keepdim=True)
    rstd = 1 / torch.sqrt(((v - mean) ** 2).mean(dim=(1, 3), keepdim=True) + EPS)
    z = (v - mean) * rstd * s["gamma"].reshape(shape[2:]) + s["beta"].reshape(shape[2:])
    stats = torch.stack([mean, rstd], -1).reshape(c["n"], c["groups"], 2)
    return _act(c["act"], z).reshape(x.shape).to(x.dtype), stats


def _norm_backward(s):
    c, x = s["case"], s["x"]
    shape = (c["n"], c["h"] * c["w"], c["groups"], c["c"] // c["groups"])
    mean, rstd = (s["stats"][..., i].reshape(c["n"], 1, c["groups"], 1) for i in (0, 1))
    gamma = s["gamma"].reshape(shape[2:])
    xhat = (x.float().reshape(shape) - mean) * rstd
    dz = s["dy"].float().reshape(shape) * _slope(c["act"], xhat * gamma + s["beta"].reshape(shape[2:]))
    dgamma, dbeta = (dz * xhat).sum(dim=(0, 1)), dz.sum(dim=(0, 1))
    v = dz * gamma
    dx = rstd * (v - v.mean(dim=(1, 3), keepdim=True) - xhat * (v * xhat).mean(dim=(1, 3), keepdim=True))
    return dx.reshape(x.shape).to(x.dtype), dgamma.reshape(-1), dbeta.reshape(-1)


def _projections(s):
    x, wg, wu = s["x"].float(), s["wg"].float(), s["wu"].float()
    g, u = x @ wg.t(), x @ wu.t()
    if s["bg"] is not None:
        g, u = g + s["bg"], u + s["bu"]
    return x, wg, wu, g, u


def _ff(s):
    _, _, _, g, u = _projections(s)
    return (_act(s["case"]["act"], g) * u).to(s["x"].dtype)


def _ff_backward(s):
    act, dt = s["case"]["act"], s["x"].dtype
    x, wg, wu, g, u = _projections(s)
    dy = s["dy"].float()
    dg, du = dy * u * _slope(act, g), dy * _act(act, g)
    out = [(dg @ wg + du @ wu).to(dt), (dg.t() @ x).to(dt), (du.t() @ x).to(dt)]
    return out + ([dg.sum(0), du.sum(0)] if s["bg"] is not None else [None, None])


def _compose(a, b):
    """Inclusive prefixes over the first axis of v -> a v + b, by doubling."""
    step = 1
    while step < a.shape[0]:
        b = torch.cat([b[:step], b[step:] + a[step:] * b[:-step]])
        a = torch.cat([a[:step], a[step:] * a[:-step]])
        step *= 2
    return a, b


def _gates(s):
    """Share of the state that a frame keeps, of the value that it takes, and which frames there are."""
    t, n = s["case"]["t"], s["case"]["n"]
    g = s["g"].float()
    keep, take = 1 / (1 + torch.exp(-g)), 1 / (1 + torch.exp(g))
    live = torch.ones(t, n, 1, dtype=torch.bool, device=g.device)
    if s["lengths"] is not None:
        live = (torch.arange(t, device=g.device)[:, None] < s["lengths"][None, :])[..., None]
    fresh = torch.zeros_like(live) if s["reset"] is None else (s["reset"] != 0)[..., None]
    return keep, take, live, fresh


def _states(s):
    """h of every frame (frames that are not there hand the state on), from the state before the first."""
    keep, take, live, fresh = _gates(s)
    one, none = torch.ones_like(keep), torch.zeros_like(keep)
    a = torch.where(live, torch.where(fresh, none, keep), one)
    b = torch.where(live, take * s["x"].float(), none)
    a, b = _compose(a, b)
    return a * s["h0"] + b


def _scan(s):
    h = _states(s)
    last = h[-1].clone()
    live = _gates(s)[2]
    return torch.where(live, h, torch.zeros_like(h)).to(s["g"].dtype), last


def _scan_backward(s):
    keep, take, live, fresh = _gates(s)
    none = torch.zeros_like(keep)
    before = torch.cat([s["h0"][None], _states(s)[:-1]])
    passed = torch.where(live, torch.where(fresh, none, keep), torch.ones_like(keep))   # of the state before a frame to the one after
    # the gradient of frame t's state: its own, and frame t+1's share; the last state's gradient comes in behind the last frame
    a = torch.cat([passed[1:], torch.ones_like(keep[:1])]).flip(0)
    b = torch.where(live, s["dh"].float(), none).flip(0)
    a, b = _compose(a, b)
    grad = (a * s["dlast"] + b).flip(0)
    x = s["x"].float()
    dg = torch.where(live, grad * keep * take * (torch.where(fresh, none, before) - x), none)
    dx = torch.where(live, grad * take, none)
    return dg.to(s["g"].dtype), dx.to(s["g"].dtype), passed[0] * grad[0]


def run(state):
    if own:
        return _own(state)
    return globals()["_" + state["case"]["op"]](state)


def work(case):
    c, e = case, _BYTES[case["dtype"]]
    if c["op"].startswith("norm"):
        v = c["n"] * c["h"] * c["w"] * c["c"]
        back = c["op"] == "norm_backward"
        return {"bytes": v * e * (3 if back else 2) + 8 * c["c"] * (2 if back else 1) + 8 * c["n"] * c["groups"], "flops": v * (20 if back else 10)}
    if c["op"].startswith("ff"):
        m, k, f, back = c["m"], c["k"], c["f"], c["op"] == "ff_backward"
        moved = (m * k + 2 * f * k) * e * (2 if back else 1) + m * f * e + (8 * f * (2 if back else 1) if c["bias"] else 0)
        return {"bytes": moved, "flops": m * k * f * (12 if back else 4)}
    v = (sum(_lengths(c)) if c["lengths"] else c["t"] * c["n"]) * c["d"]
    back = c["op"] == "scan_backward"
    moved = v * e * (5 if back else 3) + c["n"] * c["d"] * 4 * (3 if back else 2) + (c["t"] * c["n"] if c["resets"] else 0) + (4 * c["n"] if c["lengths"] else 0)
    return {"bytes": moved, "flops": v * (24 if back else 10)}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------

def _phi(name, z):
    """(value, slope) of an activation."""
    if name == "relu":
        return z.clamp_min(0), (z > 0).double()
    if name == "leaky":
        return torch.maximum(z, z / 10), torch.where(z > 0, 1.0, 0.1).double()
    if name in ("sigmoid", "silu"):
        q = torch.special.expit(z)
        return (q, q - q * q) if name == "sigmoid" else (z * q, q + z * (q - q * q))
    if name == "gelu":
        cdf = torch.special.ndtr(z)
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return z, torch.ones_like(z)


def exact(case, seed):
    s, c = prepare(case, seed), case
    op = c["op"]
    if op.startswith("norm"):
        n, g, per = c["n"], c["groups"], c["c"] // c["groups"]
        # one row a group of an image, [n * groups][values]
        by_group = lambda v: v.double().reshape(n, -1, g, per).transpose(1, 2).reshape(n * g, -1)  # noqa: E731
        by_pixel = lambda v: v.reshape(n, g, -1, per).transpose(1, 2).reshape(s["x"].shape)        # noqa: E731
        x = by_group(s["x"])
        gamma = by_group(s["gamma"].expand(n, c["h"] * c["w"], -1))
        beta = by_group(s["beta"].expand(n, c["h"] * c["w"], -1))
        if op == "norm":
            mean = x.sum(1, keepdim=True) / x.shape[1]
            rstd = ((x - mean).square().sum(1, keepdim=True) / x.shape[1] + EPS) ** -0.5
            y = _phi(c["act"], (x - mean) * rstd * gamma + beta)[0]
            return by_pixel(y), torch.cat([mean, rstd], 1).reshape(n, g, 2)
        st = s["stats"].double().reshape(n * g, 2)
        xh = (x - st[:, :1]) * st[:, 1:]
        dz = by_group(s["dy"]) * _phi(c["act"], xh * gamma + beta)[1]
        dxh = dz * gamma
        dx = st[:, 1:] * (dxh - (dxh.sum(1, keepdim=True) + xh * (dxh * xh).sum(1, keepdim=True)) / x.shape[1])
        return by_pixel(dx), by_pixel(dz * xh).sum(dim=(0, 1, 2)), by_pixel(dz).sum(dim=(0, 1, 2))
    if op.startswith("ff"):
        x, w = s["x"].double(), torch.cat([s["wg"], s["wu"]]).double()
        both = x @ w.t()
        if c["bias"]:
            both = both + torch.cat([s["bg"], s["bu"]]).double()
        gate, up = both[:, :c["f"]], both[:, c["f"]:]
        value, slope = _phi(c["act"], gate)
        if op == "ff":
            return value * up
        d = torch.cat([up * slope, value], 1) * s["dy"].double().repeat(1, 2)
        dw, db = d.t() @ x, d.sum(0)
        f = c["f"]
        return [d @ w, dw[:f], dw[f:], db[:f] if c["bias"] else None, db[f:] if c["bias"] else None]
    t, n = c["t"], c["n"]
    ends = _lengths(c) if c["lengths"] else [t] * n
    there = torch.tensor(ends, device="cuda")[:, None]
    keep, x = torch.special.expit(s["g"].double()), s["x"].double()
    hold = keep if s["reset"] is None else keep * (s["reset"] == 0).double()[..., None]
    state, states = s["h0"].double(), []
    for i in range(t):
        states.append(state)
        state = torch.where(there > i, hold[i] * state + (1 - keep[i]) * x[i], state)
    if op == "scan":
        h = torch.stack(states[1:] + [state])
        for j, e in enumerate(ends):
            h[e:, j] = 0
        return h, state
    grad, dg, dx = s["dlast"].double(), torch.zeros_like(x), torch.zeros_like(x)
    for i in reversed(range(t)):
        on = there > i
        now = grad + s["dh"][i].double()
        before = states[i] if s["reset"] is None else states[i] * (s["reset"][i] == 0).double()[:, None]
        dg[i] = torch.where(on, now * (before - x[i]) * keep[i] * (1 - keep[i]), 0.0)
        dx[i] = torch.where(on, now * (1 - keep[i]), 0.0)
        grad = torch.where(on, now * hold[i], grad)
    return dg, dx, grad
