"""Group normalisation with an activation, channels last: forward and backward against the 64-bit definition."""
import numpy as np
import pytest
import torch

import head_ref as ref
from head_ref import U32, close, half_step

pytestmark = pytest.mark.gpu

EPS = 1e-5
TYPES = [torch.float32, torch.bfloat16, torch.float16]
# (images, height, width, channels, groups): one value a group, one pixel, odd channels a group, groups wider and narrower
# than an access, more channels than threads, images for one block a few channels and for many, more images than SMs
SIZES = [(1, 4, 4, 1, 1), (2, 1, 1, 64, 4), (3, 5, 7, 6, 2), (1, 56, 56, 64, 32), (2, 9, 11, 84, 7), (5, 3, 3, 40, 40), (1, 13, 1, 21, 3),
         (2, 17, 3, 520, 1), (1, 2, 2, 4104, 2), (1, 200, 230, 64, 1), (70, 2, 9, 32, 8), (1, 1, 3000, 12, 6),
         (500, 2, 9, 64, 16), (37, 50, 60, 64, 8), (66000, 1, 2, 8, 2)]


def _rrm():
    import paper_1802_09723_b200 as rrm
    return rrm


def _inputs(size, dtype, seed=0, pad=0, affine=True, offset=1.0):
    n, h, w, c, groups = size
    r = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, h, w, c + pad, generator=r, device="cuda") * 0.7 + offset * torch.randn(c + pad, generator=r, device="cuda")
    gamma = 1 + 0.2 * torch.randn(c, generator=r, device="cuda") if affine else None
    beta = 0.2 * torch.randn(c, generator=r, device="cuda") if affine else None
    dy = torch.randn(n, h, w, c, generator=r, device="cuda").to(dtype)
    return x.to(dtype)[..., :c], gamma, beta, dy


def _z_error(x, groups, mean, rstd, gamma):
    """Bound of the error of z = (x - mean) rstd gamma + beta computed in 32 bits, per image (broadcast over the image's values).
    The group's mean is a tree of sums and merges whose depth here is under 32 roundings of values up to max|x|; the squared
    distances lose as much of theirs and rstd half of that; the rest of z is four roundings of |z|, and the exponential
    and error functions of the activation (slope below 1.2) a few more: 64 half steps of (max|x| rstd + |z|) |gamma| in all."""
    n = x.shape[0]
    top = x.double().reshape(n, -1).abs().amax(1)
    g = 1.0 if gamma is None else float(gamma.abs().max())
    scale = (2 * top * rstd.amax(1) * g + 1).reshape((n,) + (1,) * (x.dim() - 1))
    return 64 * U32 * scale


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
def test_forward_matches_the_definition(size, dtype):
    for name, pad, affine in (("none", 0, True), ("silu", 1, True), ("relu", 8, False)):
        x, gamma, beta, _ = _inputs(size, dtype, pad=pad, affine=affine)
        y, stats = _rrm().group_norm(x, size[-1], gamma, beta, eps=EPS, act=name)
        want, mean, rstd = ref.norm(x, size[-1], gamma, beta, EPS, name)
        err = _z_error(x, size[-1], mean, rstd, gamma)
        close(y, want, half_step(dtype, want) + 1.01 * err, name)
        top = x.double().abs().max()
        close(stats[..., 0], mean, 32 * U32 * top, "mean")
        # the variance's error: 32 roundings of it, and twice the mean's error times the spread
        close(stats[..., 1], rstd, rstd * (32 * U32 + 32 * U32 * top * rstd), "rstd")


@pytest.mark.parametrize("name", ["leaky", "sigmoid", "gelu"])
def test_other_activations(name):
    size = (2, 6, 5, 32, 4)
    x, gamma, beta, _ = _inputs(size, torch.float32)
    y, _ = _rrm().group_norm(x, 4, gamma, beta, eps=EPS, act=name)
    want, mean, rstd = ref.norm(x, 4, gamma, beta, EPS, name)
    close(y, want, half_step(torch.float32, want) + _z_error(x, 4, mean, rstd, gamma), name)


def test_a_mean_far_from_zero_costs_no_more_than_the_inputs_hold():
    """Values 1000 apart from zero with a spread of one, and a first pixel that is nowhere near the others."""
    x = 1000 + torch.randn(1, 64, 64, 32, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    x[:, 0, 0] = 0
    y, stats = _rrm().group_norm(x, 4, eps=EPS)
    want, mean, rstd = ref.norm(x, 4, None, None, EPS, "none")
    close(stats[..., 1], rstd, rstd * (32 * U32 + 32 * U32 * 1100 * rstd), "rstd")
    close(y, want, half_step(torch.float32, want) + _z_error(x, 4, mean, rstd, None))


def _backward_reference(x, dy, groups, gamma, beta, name):
    xs = x.double().requires_grad_()
    g = (torch.ones(x.shape[-1], device="cuda") if gamma is None else gamma).double().requires_grad_()
    b = (torch.zeros(x.shape[-1], device="cuda") if beta is None else beta).double().requires_grad_()
    y, mean, rstd = ref.norm(xs, groups, g, b, EPS, name)
    y.backward(dy.double())
    return xs.grad, g.grad, b.grad, mean.detach(), rstd.detach()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
def test_backward_matches_the_formula(size, dtype):
    for name, pad in (("none", 0), ("silu", 1), ("gelu", 8)):
        x, gamma, beta, dy = _inputs(size, dtype, seed=1, pad=pad)
        _, stats = _rrm().group_norm(x, size[-1], gamma, beta, eps=EPS, act=name)
        dx, dgamma, dbeta = _rrm().group_norm_backward(x, dy, size[-1], gamma, beta, stats, eps=EPS, act=name)
        wx, wg, wb, mean, rstd = _backward_reference(x, dy, size[-1], gamma, beta, name)
        # dx = rstd (v - m1 - xhat m2): xhat and z are off by e (as forward), v by a few half steps and the slope's change (below
        # 1.2 a unit of z), the means by no more; every term is at most |v| (1 + xhat^2) in size
        e = float(_z_error(x, size[-1], mean, rstd, gamma).max())
        v = float(dy.double().abs().max() * 1.2 * gamma.abs().max())
        xh = float(((x.double().reshape(x.shape[0], -1).amax(1) - mean.amin(1)).abs().max() + mean.abs().max()) * rstd.max())
        xh = min(xh, float(np.sqrt(x[0].numel() // size[-1])))                     # |xhat| of n values is at most sqrt(n)
        r = rstd.amax(1).reshape(-1, 1, 1, 1)
        close(dx, wx, half_step(dtype, wx) + 3 * r * v * (1 + xh) ** 2 * e, name)
        count = x.numel() // size[3]
        # a sum of `count` terms in a tree: 64 roundings of at most the sum of magnitudes, and e a term
        close(dgamma, wg, count * (1.2 * float(dy.double().abs().max())) * (1 + xh) * (e + 64 * U32 / np.sqrt(count)), "dgamma")
        close(dbeta, wb, count * (1.2 * float(dy.double().abs().max())) * (e + 64 * U32 / np.sqrt(count)), "dbeta")


@pytest.mark.parametrize("name", ["relu", "leaky"])
def test_backward_of_kinked_activations_away_from_the_kink(name):
    x, gamma, beta, dy = _inputs((2, 8, 8, 32, 4), torch.float32, seed=5)
    _, mean, rstd = ref.norm(x, 4, gamma, beta, EPS, "none")
    z = ref.norm(x, 4, gamma, beta, EPS, "none")[0]
    dy = torch.where(z.abs() < 1e-4, torch.zeros_like(dy), dy)                      # where 32 bits may fall on the other side
    _, stats = _rrm().group_norm(x, 4, gamma, beta, eps=EPS, act=name)
    dx, dgamma, dbeta = _rrm().group_norm_backward(x, dy, 4, gamma, beta, stats, act=name)
    wx, wg, wb, mean, rstd = _backward_reference(x, dy, 4, gamma, beta, name)
    e = float(_z_error(x, 4, mean, rstd, gamma).max())
    v = float(dy.abs().max() * gamma.abs().max())
    close(dx, wx, half_step(torch.float32, wx) + 3 * float(rstd.max()) * v * 36 * e)
    close(dgamma, wg, 128 * float(dy.abs().max()) * 6 * e)
    close(dbeta, wb, 128 * float(dy.abs().max()) * e)


def test_backward_agrees_with_differences():
    """Along a random direction of x, gamma and beta together, in 64 bits, the loss changes by the gradient's share of it."""
    x, gamma, beta, dy = _inputs((2, 5, 6, 24, 3), torch.float32, seed=7)
    _, stats = _rrm().group_norm(x, 3, gamma, beta, eps=EPS, act="silu")
    dx, dgamma, dbeta = _rrm().group_norm_backward(x, dy, 3, gamma, beta, stats, act="silu")
    r = torch.Generator(device="cuda").manual_seed(8)
    d = [torch.randn(t.shape, generator=r, device="cuda", dtype=torch.float64) for t in (x, gamma, beta)]

    def loss(s):
        y = ref.norm(x.double() + s * d[0], 3, gamma.double() + s * d[1], beta.double() + s * d[2], EPS, "silu")[0]
        return float((y * dy.double()).sum())

    step = 1e-4
    want = (loss(step) - loss(-step)) / (2 * step)
    got = float((dx.double() * d[0]).sum() + (dgamma.double() * d[1]).sum() + (dbeta.double() * d[2]).sum())
    # differences are off by step^2 times a third derivative, some hundreds at worst here
    assert abs(got - want) <= 1e-4 * (1 + abs(want)), (got, want)


def test_a_poisoned_group_stays_alone():
    for bad in (float("nan"), float("inf")):
        x, gamma, beta, dy = _inputs((2, 6, 6, 32, 8), torch.bfloat16, seed=9)
        x = x.contiguous()
        x[1, 3, 3, 5] = bad
        y, stats = _rrm().group_norm(x, 8, gamma, beta, act="none")
        hit = torch.zeros_like(y, dtype=torch.bool)
        hit[1, :, :, 4:8] = True
        assert not torch.isfinite(y[hit]).any()
        assert torch.isfinite(y[~hit]).all()
        dx, dgamma, _ = _rrm().group_norm_backward(x, dy, 8, gamma, beta, stats)
        assert torch.isfinite(dx[~hit]).all() and not torch.isfinite(dx[hit]).any()
        assert torch.isfinite(dgamma[torch.tensor([0, 1, 2, 3] + list(range(8, 32)), device="cuda")]).all()


def test_constant_values_and_single_values_have_no_spread():
    x = torch.full((2, 3, 3, 8), 7.0, device="cuda")
    y, stats = _rrm().group_norm(x, 2, beta=torch.arange(8.0, device="cuda"), eps=1e-2)
    assert torch.equal(y, torch.arange(8.0, device="cuda").expand_as(y))
    close(stats[..., 1], torch.full((2, 2), 10.0, dtype=torch.float64, device="cuda"), 10 * 8 * U32)


def test_in_place_strided_images_and_no_images():
    x, gamma, beta, dy = _inputs((3, 4, 4, 32, 4), torch.float16, seed=11)
    want, _ = _rrm().group_norm(x, 4, gamma, beta, act="silu")
    buf = x.contiguous().clone()
    got, _ = _rrm().group_norm(buf, 4, gamma, beta, act="silu", y=buf)
    assert got.data_ptr() == buf.data_ptr() and torch.equal(got, want)
    wide = torch.full((3, 2, 4, 4, 40), 5.0, dtype=torch.float16, device="cuda")
    out = wide[:, 0, :, :, :32]
    _rrm().group_norm(x, 4, gamma, beta, act="silu", y=out)
    assert torch.equal(out, want) and (wide[:, 1] == 5).all() and (wide[..., 32:] == 5).all()
    empty = x[:0]
    y, stats = _rrm().group_norm(empty, 4, gamma, beta)
    assert y.shape == empty.shape and stats.shape == (0, 4, 2)
    _, dgamma, dbeta = _rrm().group_norm_backward(empty, empty, 4, gamma, beta, stats)
    assert (dgamma == 0).all() and (dbeta == 0).all()


def test_offsets_beyond_32_bits():
    """Two images whose second one lies past 2^31 elements."""
    c, far = 16, (1 << 31) + 64
    buf = torch.empty(far + 4 * c, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((2, 2, 2, c), (far, 2 * c, c, 1))
    small, gamma, beta, dy = _inputs((2, 2, 2, c, 2), torch.bfloat16, seed=13)
    x.copy_(small)
    y, stats = _rrm().group_norm(x, 2, gamma, beta, act="silu")
    want, _ = _rrm().group_norm(small, 2, gamma, beta, act="silu")
    assert torch.equal(y, want)
    a = _rrm().group_norm_backward(x, dy, 2, gamma, beta, stats, act="silu")
    b = _rrm().group_norm_backward(small, dy, 2, gamma, beta, stats, act="silu")
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_another_stream_and_a_captured_call():
    x, gamma, beta, dy = _inputs((4, 16, 16, 64, 8), torch.bfloat16, seed=15)
    y, stats = _rrm().group_norm(x, 8, gamma, beta, act="silu")
    back = _rrm().group_norm_backward(x, dy, 8, gamma, beta, stats, act="silu")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y2, st2 = _rrm().group_norm(x, 8, gamma, beta, act="silu", stream=s)
    back2 = _rrm().group_norm_backward(x, dy, 8, gamma, beta, st2, act="silu", stream=s)
    s.synchronize()
    assert torch.equal(y, y2) and all(torch.equal(a, b) for a, b in zip(back, back2))
    graph = torch.cuda.CUDAGraph()
    xs = x.clone()
    with torch.cuda.graph(graph):
        y3, st3 = _rrm().group_norm(xs, 8, gamma, beta, act="silu")
        back3 = _rrm().group_norm_backward(xs, dy, 8, gamma, beta, st3, act="silu")
    for k in range(2):
        xs.copy_(x if k == 0 else x.flip(0))
        graph.replay()
        y4, st4 = _rrm().group_norm(xs, 8, gamma, beta, act="silu")
        back4 = _rrm().group_norm_backward(xs, dy, 8, gamma, beta, st4, act="silu")
        assert torch.equal(y3, y4) and all(torch.equal(a, b) for a, b in zip(back3, back4))


def test_a_stack_s_tensor_is_normalised_where_it_lies():
    import workloads as wl
    rrm = _rrm()
    specs = wl.single_conv_f32(c_in=16, c_out=24, hw=20)
    video = wl.block_redraw_sequence(frames=3, c=16, hw=20, seed=2)
    net = rrm.net_from_specs(specs)
    for t in range(3):
        net.step(torch.from_numpy(video[t]).cuda())
        x = net.tensor(1).permute(0, 2, 3, 1).contiguous()
        y, stats = net.group_norm(1, 6, act="relu")
        want, wstats = rrm.group_norm(x, 6, act="relu")
        assert torch.equal(y, want) and torch.equal(stats, wstats)
    with pytest.raises(rrm.RRMError):
        net.group_norm(1, 5)
    net.close()


def test_refusals():
    rrm = _rrm()
    x, gamma, beta, dy = _inputs((2, 4, 4, 16, 4), torch.float32)
    _, stats = rrm.group_norm(x, 4)
    for bad in (lambda: rrm.group_norm(x, 3), lambda: rrm.group_norm(x, 0), lambda: rrm.group_norm(x, 4, act="sign"),
                lambda: rrm.group_norm(x, 4, act="tanh"), lambda: rrm.group_norm(x, 4, eps=0.0), lambda: rrm.group_norm(x.double(), 4),
                lambda: rrm.group_norm(x.cpu(), 4), lambda: rrm.group_norm(x, 4, gamma=gamma.half()),
                lambda: rrm.group_norm(x, 4, gamma=gamma[:8]), lambda: rrm.group_norm(x.permute(0, 3, 1, 2), 4),
                lambda: rrm.group_norm(x.transpose(1, 2), 4), lambda: rrm.group_norm(x, 4, y=x[:1]),
                lambda: rrm.group_norm(x[:1].expand(2, 4, 4, 16), 4), lambda: rrm.group_norm_backward(x, dy, 4),
                lambda: rrm.group_norm_backward(x, dy.half(), 4, stats=stats)):
        with pytest.raises(rrm.RRMError):
            bad()
