"""The gated feed-forward block and its backward pass against the 64-bit definition."""
import ctypes

import pytest
import torch

import head_ref as ref
from head_ref import U32, close, half_step

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
# (rows, inputs, outputs): one row, one of everything, one contraction stage and parts of one, row tiles of 8, 128 and 256 and
# one more, column tiles of 32, 64 and 128 and one more, enough tiles for every width of tile and for several tiles a block;
# few rows, short and long ones, of widths that allow wide accesses and not
SIZES = [(1, 64, 64), (1, 1, 1), (1, 1500, 33), (3, 16, 8), (8, 63, 31), (9, 65, 32), (128, 128, 128), (129, 200, 129), (200, 72, 520), (257, 64, 96),
         (300, 1000, 1001), (513, 130, 640), (1100, 256, 1300), (2304, 64, 4800),
         (2, 40, 7), (4, 2050, 65), (7, 4096, 130), (5, 4096, 2050), (6, 11001, 30)]


def _rrm():
    import paper_1802_09723_b200 as rrm
    return rrm


def _inputs(size, dtype, seed=0, pad=0, bias=True, scale=1.0):
    m, k, f = size
    r = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *s, by=1.0: torch.randn(*s, generator=r, device="cuda") * by                       # noqa: E731
    x = new(m, k + pad, by=scale).to(dtype)[:, :k]
    wg, wu = (new(f, k + pad, by=k ** -0.5).to(dtype)[:, :k] for _ in range(2))
    bg, bu = (new(f, by=0.1) if bias else None for _ in range(2))
    return x, wg, wu, bg, bu, new(m, f).to(dtype)


def _sum_error(k, dtype):
    """Relative error of a sum of k products against the sum of their magnitudes: a tensor core adds 16 of them a step to an
    fp32 accumulator, cut to its 24 bits (2 half steps) with each step, and as much inside a step; fp32 makes six such passes
    and leaves out piece products of 3 * 2^-24 of each product."""
    steps = (k + 15) // 16 + 4
    return (4 * steps * U32) if dtype == BF16 else (4 * 6 * steps * U32 + 4 * U32)


def _parts(x, wg, wu, bg, bu, name, dtype):
    """Projections, activation and slope in 64 bits, and the bound of a projection's error."""
    X, G, W = x.double(), wg.double(), wu.double()
    g, u = X @ G.t(), X @ W.t()
    size = torch.maximum(X.abs() @ G.abs().t(), X.abs() @ W.abs().t())
    if bg is not None:
        g, u = g + bg.double(), u + bu.double()
        size = size + torch.maximum(bg.abs(), bu.abs()).double()
    z = g.clone().requires_grad_()
    value = ref.act(name, z)
    slope, = torch.autograd.grad(value.sum(), z)
    return g, u, value.detach(), slope, size * _sum_error(x.shape[1], dtype) + 2 * U32 * size


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", SIZES)
def test_forward_matches_the_definition(size, dtype):
    for name, pad, bias in (("silu", 0, True), ("none", 1, False), ("gelu", 8, True)):
        x, wg, wu, bg, bu, _ = _inputs(size, dtype, pad=pad, bias=bias)
        y = _rrm().gated_ff(x, wg, wu, bg, bu, act=name)
        _, u, value, _, err = _parts(x, wg, wu, bg, bu, name, dtype)
        # slope below 1.2; the activation's own exponential: 16 half steps of its value
        close(y, value * u, half_step(dtype, value * u) + 1.01 * (1.2 * err * (u.abs() + err) + (value.abs() + 1e-30) * (err + 16 * U32 * u.abs())), name)
    _rrm().head_status()


@pytest.mark.parametrize("name", ["relu", "leaky", "sigmoid"])
def test_other_activations(name):
    x, wg, wu, bg, bu, dy = _inputs((70, 100, 90), F32, seed=1)
    y = _rrm().gated_ff(x, wg, wu, bg, bu, act=name)
    g, u, value, slope, err = _parts(x, wg, wu, bg, bu, name, F32)
    close(y, value * u, half_step(F32, y.double()) + 1.2 * err * (u.abs() + err) + value.abs() * (err + 16 * U32 * u.abs()), name)
    dy = torch.where(g.abs() < 1e-3, torch.zeros_like(dy), dy)                      # where 32 bits may fall on a kink's other side
    back = _rrm().gated_ff_backward(x, wg, wu, dy, bg, bu, act=name)
    _check_backward(back, x, wg, wu, bg, bu, dy, name, F32)


def _check_backward(got, x, wg, wu, bg, bu, dy, name, dtype):
    g, u, value, slope, err = _parts(x, wg, wu, bg, bu, name, dtype)
    D = dy.double()
    dg, du = D * u * slope, D * value
    # slope and value move by at most 1.2 a unit of g; 32 half steps for the exponentials
    eg = D.abs() * (err * (slope.abs() + 1.2 * u.abs() + 1.2 * err) + 32 * U32 * u.abs() * (slope.abs() + 1))
    eu = D.abs() * (1.2 * err + 32 * U32 * (value.abs() + 1))
    m, k = x.shape
    # dg and du on their way to the last products: one rounding to bf16, or three pieces
    if dtype == BF16:
        rg, ru = eg + half_step(BF16, dg) + eg * 2 ** -8, eu + half_step(BF16, du) + eu * 2 ** -8
    else:
        rg, ru = eg + U32 * dg.abs(), eu + U32 * du.abs()
    X, G, W = x.double(), wg.double(), wu.double()
    dx, dwg, dwu = dg @ G + du @ W, dg.t() @ X, du.t() @ X
    sum_x = (dg.abs() + rg) @ G.abs() + (du.abs() + ru) @ W.abs()
    close(got[0], dx, half_step(dtype, dx) + 1.01 * (rg @ G.abs() + ru @ W.abs() + sum_x * _sum_error(2 * wg.shape[0], dtype)), "dx")
    for i, (d, r, want) in enumerate(((dg, rg, dwg), (du, ru, dwu))):
        size = (d.abs() + r).t() @ X.abs()
        close(got[1 + i], want, half_step(dtype, want) + 1.01 * (r.t() @ X.abs() + size * _sum_error(m, dtype)), "dw")
    if bg is not None:
        close(got[3], dg.sum(0), eg.sum(0) + dg.abs().sum(0) * 16 * U32 + m / 32 * U32 * dg.abs().sum(0), "dbg")
        close(got[4], du.sum(0), eu.sum(0) + du.abs().sum(0) * 16 * U32 + m / 32 * U32 * du.abs().sum(0), "dbu")
    else:
        assert got[3] is None and got[4] is None


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", SIZES)
def test_backward_matches_the_formula(size, dtype):
    for name, pad, bias in (("silu", 0, True), ("gelu", 1, False)):
        x, wg, wu, bg, bu, dy = _inputs(size, dtype, seed=2, pad=pad, bias=bias)
        _check_backward(_rrm().gated_ff_backward(x, wg, wu, dy, bg, bu, act=name), x, wg, wu, bg, bu, dy, name, dtype)
    _rrm().head_status()


def test_backward_agrees_with_differences():
    x, wg, wu, bg, bu, dy = _inputs((20, 24, 30), F32, seed=3)
    got = _rrm().gated_ff_backward(x, wg, wu, dy, bg, bu, act="silu")
    r = torch.Generator(device="cuda").manual_seed(4)
    args = (x, wg, wu, bg, bu)
    d = [torch.randn(t.shape, generator=r, device="cuda", dtype=torch.float64) for t in args]

    def loss(s):
        return float((ref.gated_ff(*(t.double() + s * e for t, e in zip(args, d)), "silu") * dy.double()).sum())

    step = 1e-4
    want = (loss(step) - loss(-step)) / (2 * step)
    have = sum(float((a.double() * b).sum()) for a, b in zip(got, d))
    assert abs(have - want) <= 1e-4 * (1 + abs(want)), (have, want)


def test_fp32_keeps_small_and_large_values():
    """Rows many powers of two apart, and weights the other way: each row's products keep fp32's digits."""
    x, wg, wu, _, _, _ = _inputs((40, 96, 64), F32, seed=5, bias=False)
    power = 2.0 ** (torch.arange(40, device="cuda") % 13 * 5 - 30).float()[:, None]
    y = _rrm().gated_ff(x * power, wg, wu, act="none")
    _, u, value, _, err = _parts(x * power, wg, wu, None, None, "none", F32)
    close(y, value * u, half_step(F32, value * u) + 1.01 * (err * (u.abs() + err) + value.abs() * (err + 4 * U32 * u.abs())))
    big = torch.full((1, 4), 3.4e38, device="cuda")                                 # beyond bf16's largest value, 3.39e38
    w = torch.zeros(2, 4, device="cuda")
    w[:, 0] = 1.0
    wu = torch.zeros(2, 4, device="cuda")
    wu[:, 0] = 2.0 ** -20
    y = _rrm().gated_ff(big * 2.0 ** -100, w, wu, act="none")
    z = big[0, 0].double() * 2.0 ** -100
    close(y, (z * z * 2.0 ** -20).expand(1, 2), float(z * z * 2.0 ** -20) * 32 * U32)
    y = _rrm().gated_ff(big, w * 2.0 ** -64, wu * 2.0 ** -64, act="none")
    z = big[0, 0].double() * 2.0 ** -64
    close(y, (z * z * 2.0 ** -20).expand(1, 2), float(z * z * 2.0 ** -20) * 32 * U32)


def test_values_that_are_not_finite_stay_in_their_row_or_column():
    for dtype in (F32, BF16):
        x, wg, wu, bg, bu, dy = (t.clone() for t in _inputs((150, 96, 140), dtype, seed=6))
        x[7, 3] = float("nan")
        wg[9, 5] = float("inf")
        y = _rrm().gated_ff(x, wg, wu, bg, bu, act="none")
        hit = torch.zeros_like(y, dtype=torch.bool)
        hit[7], hit[:, 9] = True, True
        assert torch.isfinite(y[~hit]).all() and not torch.isfinite(y[hit]).any()


def test_rows_between_and_behind_are_left_alone():
    for dtype in (F32, BF16):
        x, wg, wu, bg, bu, _ = _inputs((37, 70, 45), dtype, seed=7)
        want = _rrm().gated_ff(x, wg, wu, bg, bu)
        wide = torch.full((40, 61), 5.0, dtype=dtype, device="cuda")
        _rrm().gated_ff(x, wg, wu, bg, bu, y=wide[:37, 3:48])
        assert torch.equal(wide[:37, 3:48], want)
        assert (wide[37:] == 5).all() and (wide[:, :3] == 5).all() and (wide[:, 48:] == 5).all()


def test_misaligned_operands_and_leading_axes():
    """Operands on element boundaries only are copied first; the leading axes of x are rows."""
    m, k, f = 30, 64, 48
    x, wg, wu, bg, bu, dy = _inputs((m, k, f), BF16, seed=8)
    want = _rrm().gated_ff(x, wg, wu, bg, bu)
    back = _rrm().gated_ff_backward(x, wg, wu, dy, bg, bu)
    off = lambda t: torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")[1:].view(t.shape).copy_(t)      # noqa: E731
    assert torch.equal(_rrm().gated_ff(off(x), off(wg), off(wu), bg, bu), want)
    assert all(torch.equal(a, b) for a, b in zip(_rrm().gated_ff_backward(off(x), off(wg), off(wu), off(dy), bg, bu), back))
    y = _rrm().gated_ff(x.view(5, 2, 3, k), wg, wu, bg, bu)
    assert y.shape == (5, 2, 3, f) and torch.equal(y.view(m, f), want)
    assert torch.equal(_rrm().gated_ff(x[4], wg, wu, bg, bu), _rrm().gated_ff(x[4:5], wg, wu, bg, bu)[0])
    both = torch.cat([wg, wu])                                                       # one parameter's halves
    assert torch.equal(_rrm().gated_ff(x, both[:f], both[f:], bg, bu), want)


def test_no_rows():
    x, wg, wu, bg, bu, dy = _inputs((4, 32, 24), BF16, seed=9)
    assert _rrm().gated_ff(x[:0], wg, wu, bg, bu).shape == (0, 24)
    dx, dwg, dwu, dbg, dbu = _rrm().gated_ff_backward(x[:0], wg, wu, dy[:0], bg, bu)
    assert dx.shape == (0, 32) and all((t == 0).all() for t in (dwg, dwu, dbg, dbu))


def test_offsets_beyond_32_bits():
    """Rows so far apart that the last ones lie past 2^31 elements."""
    m, k, f, far = 3, 64, 40, (1 << 30) + 64
    buf = torch.empty(2 * far + 64, dtype=BF16, device="cuda")
    x = buf.as_strided((m, k), (far, 1))
    small, wg, wu, bg, bu, dy = _inputs((m, k, f), BF16, seed=10)
    x.copy_(small)
    assert torch.equal(_rrm().gated_ff(x, wg, wu, bg, bu), _rrm().gated_ff(small, wg, wu, bg, bu))
    out = buf.as_strided((m, f), (far, 1))
    assert torch.equal(_rrm().gated_ff(small, wg, wu, bg, bu, y=out), _rrm().gated_ff(small, wg, wu, bg, bu))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_streams_captures_and_the_same_bits_again(dtype):
    x, wg, wu, bg, bu, dy = _inputs((300, 250, 700), dtype, seed=11)
    fwd = lambda **kw: (_rrm().gated_ff(x, wg, wu, bg, bu, **kw),)                   # noqa: E731
    bwd = lambda **kw: _rrm().gated_ff_backward(x, wg, wu, dy, bg, bu, **kw)         # noqa: E731
    first = fwd() + bwd()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = fwd(stream=s) + bwd(stream=s)
    again = fwd() + bwd()
    s.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(first, other, again))
    graphs, outs = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(fwd() + bwd())
        graphs.append(graph)
    graphs[0].replay()
    with torch.cuda.stream(s):
        graphs[1].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for o in outs for a, b in zip(first, o))


def test_refusals():
    rrm = _rrm()
    x, wg, wu, bg, bu, dy = _inputs((6, 32, 24), BF16)
    for bad in (lambda: rrm.gated_ff(x, wg, wu[:8]), lambda: rrm.gated_ff(x[:, :16], wg, wu), lambda: rrm.gated_ff(x.half(), wg.half(), wu.half()),
                lambda: rrm.gated_ff(x, wg.float(), wu), lambda: rrm.gated_ff(x, wg, wu, act="sign"), lambda: rrm.gated_ff(x, wg, wu, act="swish"),
                lambda: rrm.gated_ff(x, wg, wu, bg.half(), bu), lambda: rrm.gated_ff(x, wg, wu, bg[:3], bu), lambda: rrm.gated_ff(x.cpu(), wg, wu),
                lambda: rrm.gated_ff(x, wg.t().contiguous().t(), wu), lambda: rrm.gated_ff(x, wg, wu, y=dy[:3]),
                lambda: rrm.gated_ff(x, wg[:0], wu[:0]), lambda: rrm.gated_ff(x[:1].expand(6, 32), wg, wu),
                lambda: rrm.gated_ff_backward(x, wg, wu, dy[:, :8]), lambda: rrm.gated_ff_backward(x, wg, wu, dy.float())):
        with pytest.raises(rrm.RRMError):
            bad()


def test_a_wait_that_runs_out_is_reported_and_leaves_the_context_usable():
    """wait_limit < 0: every role of a block meets its first wait before it has issued anything and leaves."""
    rrm = _rrm()
    x, wg, wu, bg, bu, _ = _inputs((300, 256, 640), BF16, seed=12)
    want = rrm.gated_ff(x, wg, wu, bg, bu)
    rrm.head_status()
    for m in (5, 300):
        d = rrm.FfDesc()
        d.dtype, d.act, d.m, d.k, d.f, d.wait_limit = rrm.DTYPE["bf16"], rrm.ACT["silu"], m, 256, 640, -1
        y = torch.empty(m, 640, dtype=BF16, device="cuda")
        status = rrm.lib().rrm_gated_ff(ctypes.byref(d), x.data_ptr(), wg.data_ptr(), wu.data_ptr(), bg.data_ptr(), bu.data_ptr(),
                                        y.data_ptr(), None, 0, torch.cuda.current_stream().cuda_stream)
        assert status == 0
        with pytest.raises(rrm.RRMError):
            rrm.head_status()
        rrm.head_status()
    assert torch.equal(rrm.gated_ff(x, wg, wu, bg, bu), want)
    rrm.head_status()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [(1, 4096, 200), (3, 333, 65), (8, 256, 128)])
def test_few_rows_leave_what_is_beside_them(size, dtype):
    """Rows, columns and padding that are not the call's keep their values, a row that is not finite stays one row, and a captured
    call gives what the eager one gives."""
    m, k, f = size
    x, wg, wu, bg, bu, _ = _inputs(size, dtype, seed=21, pad=8)
    room = torch.full((m + 2, f + 5), 7.0, dtype=dtype, device="cuda")
    y = room[1:m + 1, 2:f + 2]
    want = _rrm().gated_ff(x, wg, wu, bg, bu)
    _rrm().gated_ff(x, wg, wu, bg, bu, y=y)
    assert torch.equal(y, want)
    outside = torch.ones_like(room, dtype=torch.bool)
    outside[1:m + 1, 2:f + 2] = False
    assert (room[outside] == 7).all()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        again = _rrm().gated_ff(x, wg, wu, bg, bu)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(again, want)
    if m > 1:
        bad = x.clone()
        bad[1, k // 2] = float("nan")
        got = _rrm().gated_ff(bad, wg, wu, bg, bu)
        keep = [i for i in range(m) if i != 1]
        assert torch.isnan(got[1]).all()
        want2 = _rrm().gated_ff(bad.nan_to_num(0.0), wg, wu, bg, bu)
        assert torch.equal(got[keep], want2[keep])
