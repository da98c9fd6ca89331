"""The head operators as they are used together: a stack's feature maps, normalised, through the gated block into the gated
recurrence, frame by frame and as a chunk, and the gradients of the whole head."""
import numpy as np
import pytest
import torch

import workloads as wl
import head_ref as ref

pytestmark = pytest.mark.gpu

GROUPS, D, EPS = 4, 12, 1e-5


def _rrm():
    import paper_1802_09723_b200 as rrm
    return rrm


def _stack(frames):
    specs = wl.single_conv_f32(c_in=8, c_out=16, hw=10)
    video = wl.block_redraw_sequence(frames=frames, c=8, hw=10, seed=2)
    return _rrm().net_from_specs(specs), [torch.from_numpy(video[t]).cuda() for t in range(frames)]


def _parameters(k, seed=0):
    r = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *s, by=1.0: torch.randn(*s, generator=r, device="cuda") * by       # noqa: E731
    return dict(gamma=1 + new(16, by=0.1), beta=new(16, by=0.1), wg=new(2 * D, k, by=k ** -0.5), wu=new(2 * D, k, by=k ** -0.5),
                bg=new(2 * D, by=0.1), bu=new(2 * D, by=0.1))


def _features(net, frames, p):
    """Normalised maps [frames][1][pixels * channels] of every frame, and their statistics."""
    rows, stats = [], []
    for f in frames:
        net.step(f)
        y, st = net.group_norm(1, GROUPS, p["gamma"], p["beta"], eps=EPS, act="silu")
        rows.append(y.reshape(1, 1, -1))
        stats.append(st)
    return torch.cat(rows), torch.cat(stats)


def test_a_frame_at_a_time_gives_what_the_chunk_gives():
    """A keyframe in the middle resets the recurrence with the stack; the serving form keeps one state buffer."""
    rrm = _rrm()
    net, frames = _stack(9)
    p = _parameters(10 * 10 * 16)
    cut = 5
    reset = torch.zeros(9, 1, dtype=torch.uint8, device="cuda")
    reset[cut] = 1
    feats, _ = _features(net, frames, p)
    proj = rrm.gated_ff(feats, p["wg"], p["wu"], p["bg"], p["bu"])
    h, last = rrm.gated_scan(proj[..., :D], proj[..., D:], reset=reset)
    # the same, a frame per call, the stack keyframed at the cut
    net2, _ = _stack(9)
    state = torch.zeros(1, D, device="cuda")
    for t, f in enumerate(frames):
        (net2.keyframe if t == cut else net2.step)(f)
        y, _ = net2.group_norm(1, GROUPS, p["gamma"], p["beta"], eps=EPS, act="silu")
        pr = rrm.gated_ff(y.reshape(1, 1, -1), p["wg"], p["wu"], p["bg"], p["bu"])
        ht, _ = rrm.gated_scan(pr[..., :D], pr[..., D:], state, reset=reset[t:t + 1], last=state)
        # the convolutions agree to 1e-4 of their largest value, and no later step enlarges that by more than ten
        assert float((ht[0] - h[t]).abs().max()) <= 1e-3 * float(h.abs().max()), t
    assert float((state - last).abs().max()) <= 1e-3 * float(h.abs().max())
    rrm.head_status()
    net.close()
    net2.close()


def _reference(x, p, reset, weight):
    """Loss and gradients in 64 bits, of the convolution's maps x [frames, h, w, c] on."""
    q = {k: v.double().requires_grad_() for k, v in p.items()}
    x = x.double().requires_grad_()
    y, _, _ = ref.norm(x, GROUPS, q["gamma"], q["beta"], EPS, "silu")
    proj = ref.gated_ff(y.reshape(x.shape[0], 1, -1), q["wg"], q["wu"], q["bg"], q["bu"], "silu")
    h, last = ref.scan(proj[..., :D], proj[..., D:], None, reset, None)
    loss = (h * weight.double()).sum() + last.sum()
    keys = list(q)
    grads = torch.autograd.grad(loss, [x] + [q[k] for k in keys])
    return loss.item(), grads[0], dict(zip(keys, grads[1:]))


def test_the_head_s_gradients():
    rrm = _rrm()
    T = 7
    net, frames = _stack(T)
    p = _parameters(10 * 10 * 16, seed=1)
    maps = []
    for f in frames:
        net.step(f)
        maps.append(net.tensor(1).permute(0, 2, 3, 1))
    net.close()
    x = torch.cat(maps).contiguous()
    reset = torch.zeros(T, 1, dtype=torch.uint8, device="cuda")
    reset[3] = 1
    weight = torch.randn(T, 1, D, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")

    y, stats = rrm.group_norm(x, GROUPS, p["gamma"], p["beta"], eps=EPS, act="silu")
    feats = y.reshape(T, 1, -1)
    proj = rrm.gated_ff(feats, p["wg"], p["wu"], p["bg"], p["bu"])
    h, last = rrm.gated_scan(proj[..., :D], proj[..., D:], reset=reset)
    dproj = torch.empty_like(proj)                                       # its halves are written in place
    rrm.gated_scan_backward(proj[..., :D], proj[..., D:], weight, None, torch.ones(1, D, device="cuda"), reset=reset,
                            dg=dproj[..., :D], dx=dproj[..., D:])
    dfeats, dwg, dwu, dbg, dbu = rrm.gated_ff_backward(feats, p["wg"], p["wu"], dproj, p["bg"], p["bu"])
    dx, dgamma, dbeta = rrm.group_norm_backward(x, dfeats.reshape(x.shape), GROUPS, p["gamma"], p["beta"], stats, eps=EPS, act="silu")

    loss, wx, want = _reference(x, p, reset, weight)
    got = dict(gamma=dgamma, beta=dbeta, wg=dwg, wu=dwu, bg=dbg, bu=dbu)
    # six steps in fp32, each off by less than 2e-5 of its largest value at these sizes (their own tests), none of which is enlarged
    # by a later one's by more than the next one's own size: 2e-4 of a gradient's largest value
    for k in want:
        assert float((got[k].double() - want[k]).abs().max()) <= 2e-4 * float(want[k].abs().max()), k
    assert float((dx.double() - wx).abs().max()) <= 2e-4 * float(wx.abs().max())

    # and against differences of the loss along the gradient itself: step^2 times a third derivative is far below a thousandth here
    step = 1e-4 / max(float(v.abs().max()) for v in want.values())
    moved = [_reference(x, {k: v.double() + s * step * got[k].double() for k, v in p.items()}, reset, weight)[0] for s in (1, -1)]
    slope = sum(float(v.double().square().sum()) for v in got.values())
    assert abs((moved[0] - moved[1]) / (2 * step) - slope) <= 1e-3 * slope
    assert abs(float((h * weight).sum() + last.sum()) - loss) <= 2e-4 * float(h.abs().max() * weight.abs().sum())


def test_two_training_steps_as_a_graph():
    """Forward and backward passes captured once and replayed on new inputs give what eager calls give."""
    rrm = _rrm()
    T, n, k = 33, 3, 96
    r = torch.Generator(device="cuda").manual_seed(5)
    new = lambda *s, by=1.0: (torch.randn(*s, generator=r, device="cuda") * by).bfloat16()            # noqa: E731
    wg, wu = new(2 * D * 4, k, by=0.1), new(2 * D * 4, k, by=0.1)
    x, dh = new(T, n, k), new(T, n, 4 * D)

    def step():
        proj = rrm.gated_ff(x, wg, wu)
        g, v = proj[..., :4 * D], proj[..., 4 * D:]
        h, last = rrm.gated_scan(g, v)
        dproj = torch.empty_like(proj)
        rrm.gated_scan_backward(g, v, dh, dg=dproj[..., :4 * D], dx=dproj[..., 4 * D:])
        return (h, last) + rrm.gated_ff_backward(x, wg, wu, dproj)[:3]

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for _ in range(2):
        x.copy_(new(T, n, k))
        dh.copy_(new(T, n, 4 * D))
        graph.replay()
        for a, b in zip(outs, step()):
            assert torch.equal(a, b)
