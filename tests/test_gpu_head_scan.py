"""The gated recurrence over frames: forward, backward and the step of one frame against the 64-bit definition."""
import numpy as np
import pytest
import torch

import head_ref as ref
from head_ref import U32, close, half_step

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
# (frames, streams, features): pieces of 8 and 16 frames, blocks of 64 and 128, clusters of 512 and 1024, and one more or less
SIZES = [(1, 1, 1), (1, 4, 512), (2, 3, 33), (7, 1, 4), (8, 2, 130), (9, 2, 132), (16, 1, 31), (17, 3, 5), (63, 2, 64), (64, 1, 128), (65, 2, 8),
         (129, 1, 7), (257, 2, 12), (511, 1, 4), (512, 1, 132), (513, 2, 4), (1024, 1, 3), (1025, 2, 5), (1100, 2, 260), (4200, 1, 9)]


def _rrm():
    import paper_1802_09723_b200 as rrm
    return rrm


def _inputs(size, dtype, seed=0, packed=False, resets=True, lengths=True):
    T, n, d = size
    r = torch.Generator(device="cuda").manual_seed(seed)
    both = torch.randn(T, n, 2 * d, generator=r, device="cuda")
    both[..., :d] = (both[..., :d] + 2).clamp(-6, 6)
    both = both.to(dtype)
    g, x = both[..., :d], both[..., d:]
    if not packed:
        g, x = g.contiguous(), x.contiguous()
    h0 = torch.randn(n, d, generator=r, device="cuda")
    reset = (torch.rand(T, n, generator=r, device="cuda") < 0.05).to(torch.uint8) if resets else None
    lens = torch.tensor([T - i * T // (2 * n) for i in range(n)], dtype=torch.int32, device="cuda") if lengths else None
    dh = torch.randn(T, n, d, generator=r, device="cuda").to(dtype)
    dlast = torch.randn(n, d, generator=r, device="cuda")
    return g, x, h0, reset, lens, dh, dlast


def _memory(g):
    """How many frames' errors add up in a state at most: the states' share that a frame keeps, f, is at most fmax."""
    f = float(torch.sigmoid(g.double()).max()) if g.numel() else 0.0
    return min(g.shape[0] + 1, 1 / (1 - f) + 1)


# a gate is exp (error 2 + 1.2 |g| / 2 units), a sum, a division (2 units) and a product; with |g| <= 6 and the step's product and
# sum that stays below 16 half steps of the state's size a frame
STEP = 16 * U32


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
def test_forward_matches_the_definition(size, dtype):
    for packed, resets, lengths in ((False, False, False), (True, True, True)):
        g, x, h0, reset, lens, _, _ = _inputs(size, dtype, packed=packed, resets=resets, lengths=lengths)
        h, last = _rrm().gated_scan(g, x, h0, reset=reset, lengths=lens)
        want, wlast = ref.scan(g, x, h0, reset, lens)
        top = max(float(x.abs().max()), float(h0.abs().max()))
        err = STEP * top * _memory(g)
        close(h, want, half_step(dtype, want) + err, "h")
        close(last, wlast, err, "last")


def _backward_reference(g, x, h0, reset, lens, dh, dlast):
    g, x, h0 = (t.double().requires_grad_() for t in (g, x, h0))
    h, last = ref.scan(g, x, h0, reset, lens)
    loss = (h * dh.double()).sum() + (last * dlast.double()).sum()
    return torch.autograd.grad(loss, (g, x, h0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [s for s in SIZES if s[0] <= 1100])
def test_backward_matches_the_formula(size, dtype):
    for packed, resets, lengths in ((True, False, False), (False, True, True)):
        g, x, h0, reset, lens, dh, dlast = _inputs(size, dtype, seed=1, packed=packed, resets=resets, lengths=lengths)
        dg, dx, dh0 = _rrm().gated_scan_backward(g, x, dh, h0, dlast, reset=reset, lengths=lens)
        wg, wx, wh = _backward_reference(g, x, h0, reset, lens, dh, dlast)
        m = _memory(g)
        top = max(float(x.abs().max()), float(h0.abs().max()))
        grad = float(dh.abs().max()) * m + float(dlast.abs().max())                # no gradient of a state is larger
        close(dx, wx, half_step(dtype, wx) + STEP * grad * m, "dx")
        close(dg, wg, half_step(dtype, wg) + 2 * STEP * grad * m * 2 * top, "dg")
        close(dh0, wh, STEP * grad * m, "dh0")


def test_long_backward_matches_the_formula():
    """Several chunks of a cluster's frames, wide and narrow accesses, against the analytic sums in 64 bits."""
    for d in (8, 3):
        g, x, h0, reset, lens, dh, dlast = _inputs((4200, 2, d), torch.float32, seed=2)
        dg, dx, dh0 = _rrm().gated_scan_backward(g, x, dh, h0, dlast, reset=reset, lengths=lens)
        g64, x64 = g.double(), x.double()
        f, take = torch.sigmoid(g64), torch.sigmoid(-g64)
        h, _ = ref.scan(g, x, h0, reset, lens)
        c = dlast.double()
        m = _memory(g)
        grad_top = float(dh.abs().max()) * m + float(dlast.abs().max())
        for t in reversed(range(g.shape[0])):
            on = (t < lens)[:, None]
            drop = reset[t].bool()[:, None]
            before = torch.where(drop, torch.zeros_like(c), h0.double() if t == 0 else h[t - 1])
            grad = c + dh[t].double()
            wx = torch.where(on, grad * take[t], torch.zeros_like(c))
            wg = torch.where(on, grad * f[t] * take[t] * (before - x64[t]), torch.zeros_like(c))
            if t % 97 == 0 or t > 4100 or t < 40:
                close(dx[t], wx, half_step(torch.float32, wx) + STEP * grad_top * m, f"dx {t}")
                close(dg[t], wg, half_step(torch.float32, wg) + 2 * STEP * grad_top * m * 10, f"dg {t}")
            c = torch.where(on, torch.where(drop, torch.zeros_like(c), f[t] * grad), c)
        close(dh0, c, STEP * grad_top * m, "dh0")


def test_backward_agrees_with_differences():
    g, x, h0, reset, lens, dh, dlast = _inputs((40, 2, 6), torch.float32, seed=3)
    dg, dx, dh0 = _rrm().gated_scan_backward(g, x, dh, h0, dlast, reset=reset, lengths=lens)
    r = torch.Generator(device="cuda").manual_seed(4)
    d = [torch.randn(t.shape, generator=r, device="cuda", dtype=torch.float64) for t in (g, x, h0)]

    def loss(s):
        h, last = ref.scan(g.double() + s * d[0], x.double() + s * d[1], h0.double() + s * d[2], reset, lens)
        return float((h * dh.double()).sum() + (last * dlast.double()).sum())

    step = 1e-4
    want = (loss(step) - loss(-step)) / (2 * step)
    got = sum(float((a.double() * b).sum()) for a, b in zip((dg, dx, dh0), d))
    assert abs(got - want) <= 1e-4 * (1 + abs(want)), (got, want)


def test_frames_one_at_a_time_give_the_chunk_s_states():
    """The serving form: the state is kept in one buffer and every frame is a call."""
    g, x, h0, reset, _, _, _ = _inputs((70, 3, 40), torch.bfloat16, seed=5, lengths=False)
    h, last = _rrm().gated_scan(g, x, h0, reset=reset)
    state = h0.clone()
    for t in range(70):
        ht, out = _rrm().gated_scan(g[t:t + 1], x[t:t + 1], state, reset=reset[t:t + 1], last=state)
        assert out.data_ptr() == state.data_ptr()
        close(ht[0], h[t].double(), 2 * half_step(torch.bfloat16, h[t].double()) + 2 * STEP * 5 * _memory(g), f"frame {t}")
    close(state, last.double(), 2 * STEP * 5 * _memory(g))
    # chunks of other lengths, the state in place as well
    state = h0.clone()
    for a, b in ((0, 9), (9, 64), (64, 70)):
        _rrm().gated_scan(g[a:b], x[a:b], state, reset=reset[a:b], last=state)
    close(state, last.double(), 2 * STEP * 5 * _memory(g))


def test_state_in_place_over_several_chunks():
    for d in (8, 3):
        g, x, h0, _, lens, _, _ = _inputs((2100, 2, d), torch.float32, seed=6, resets=False)
        _, last = _rrm().gated_scan(g, x, h0, lengths=lens)
        state = h0.clone()
        _rrm().gated_scan(g, x, state, lengths=lens, last=state)
        assert torch.equal(state, last)


@pytest.mark.parametrize("T", [5, 90, 700, 2500])
def test_a_reset_drops_whatever_came_before(T):
    """Infinities and NaNs before a cut do not reach the frames after it, whether a gate or the state holds them."""
    for d in (8, 3):
        g, x, h0, _, _, dh, dlast = _inputs((T, 2, d), torch.float32, seed=7, resets=False, lengths=False)
        cut = T // 2
        reset = torch.zeros(T, 2, dtype=torch.bool, device="cuda")
        reset[cut] = True
        want, wlast = _rrm().gated_scan(g, x, h0, reset=reset)
        wback = _rrm().gated_scan_backward(g, x, dh, h0, dlast, reset=reset)
        h0[0, 0] = float("inf")
        x[cut - 1, 1, 2] = float("nan")
        g[cut - 1, 0, 1] = float("nan")
        h, last = _rrm().gated_scan(g, x, h0, reset=reset)
        assert torch.equal(h[cut:], want[cut:]) and torch.equal(last, wlast)
        assert torch.isinf(h[0, 0, 0]) and torch.isnan(h[cut - 1, 1, 2])
        dg, dx, _ = _rrm().gated_scan_backward(g, x, dh, h0, dlast, reset=reset)
        assert torch.equal(dg[cut:], wback[0][cut:]) and torch.equal(dx[cut:], wback[1][cut:])
        # a gradient that is not finite behind the cut does not reach the frames before it
        g, x, h0, _, _, dh, dlast = _inputs((T, 2, d), torch.float32, seed=7, resets=False, lengths=False)
        dh[cut, 0, 0] = float("inf")
        dlast[1, 1] = float("nan")
        dg, dx, dh0 = _rrm().gated_scan_backward(g, x, dh, h0, dlast, reset=reset)
        assert torch.equal(dg[:cut], wback[0][:cut]) and torch.equal(dx[:cut], wback[1][:cut]) and torch.equal(dh0, wback[2])


def test_gates_at_the_ends_of_their_range():
    """Closed and open gates (infinite, the type's largest and lowest value) take the new value or keep the state exactly."""
    for dtype in TYPES:
        top = torch.finfo(dtype).max
        g = torch.tensor([-top, top, float("-inf"), float("inf")], device="cuda", dtype=dtype).reshape(4, 1, 1).expand(4, 1, 8).contiguous()
        x = torch.arange(1, 5, device="cuda", dtype=dtype).reshape(4, 1, 1).expand(4, 1, 8).contiguous()
        h, last = _rrm().gated_scan(g, x, torch.full((1, 8), 9.0, device="cuda"))
        assert h[:, 0, 0].tolist() == [1, 1, 3, 3] and (last == 3).all()
        dg, dx, dh0 = _rrm().gated_scan_backward(g, x, torch.ones_like(g), None, torch.ones(1, 8, device="cuda"))
        assert (dg == 0).all() and dx[:, 0, 0].tolist() == [2, 0, 3, 0] and (dh0 == 0).all()


def test_rows_behind_a_stream_s_last_frame_are_neither_read_nor_written():
    for T, d in ((6, 4), (200, 8), (1500, 3)):
        g, x, h0, reset, _, dh, dlast = _inputs((T, 4, d), torch.bfloat16, seed=8)
        lens = torch.tensor([T, 0, T // 2, 1], dtype=torch.int32, device="cuda")
        want, wlast = ref.scan(g, x, h0, reset, lens)
        for t in (g, x, dh):
            for i in range(4):
                t[int(lens[i]):, i] = float("nan")
        h = torch.full_like(g, 77)
        _, last = _rrm().gated_scan(g, x, h0, reset=reset, lengths=lens, h=h)
        dg, dx = torch.full_like(g, 78), torch.full_like(g, 79)
        _, _, dh0 = _rrm().gated_scan_backward(g, x, dh, h0, dlast, reset=reset, lengths=lens, dg=dg, dx=dx)
        for i in range(4):
            k = int(lens[i])
            assert (h[k:, i] == 77).all() and (dg[k:, i] == 78).all() and (dx[k:, i] == 79).all()
            assert torch.isfinite(h[:k, i]).all() and torch.isfinite(dg[:k, i]).all() and torch.isfinite(dx[:k, i]).all()
        close(last, wlast, STEP * 5 * _memory(torch.zeros(T, 1, 1) + 6))
        assert torch.equal(last[1], h0[1]) and torch.equal(dh0[1], dlast[1])
    # lengths outside [0, frames] count as the nearer end; no frames at all hand the state on
    g, x, h0, _, _, _, dlast = _inputs((5, 2, 4), torch.float32, seed=9, resets=False)
    a, la = _rrm().gated_scan(g, x, h0, lengths=torch.tensor([99, -3], dtype=torch.int32, device="cuda"))
    b, lb = _rrm().gated_scan(g, x, h0)
    assert torch.equal(a[:, 0], b[:, 0]) and torch.equal(la[0], lb[0]) and torch.equal(la[1], h0[1]) and (a[:, 1] == 0).all()
    none, same = _rrm().gated_scan(g[:0], x[:0], h0)
    assert none.shape[0] == 0 and torch.equal(same, h0)
    assert torch.equal(_rrm().gated_scan_backward(g[:0], x[:0], g[:0], h0, dlast)[2], dlast)


def test_offsets_beyond_32_bits_and_misaligned_rows():
    T, n, d, far = 3, 2, 8, (1 << 30) + 64
    buf = torch.empty(2 * far + 64, dtype=torch.bfloat16, device="cuda")
    g0, x0, h0, _, _, dh, dlast = _inputs((T, n, d), torch.bfloat16, seed=10, resets=False, lengths=False)
    g = buf.as_strided((T, n, d), (far, 2 * d, 1))
    x = buf[d:].as_strided((T, n, d), (far, 2 * d, 1))
    g.copy_(g0)
    x.copy_(x0)
    a, b = _rrm().gated_scan(g, x, h0), _rrm().gated_scan(g0, x0, h0)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    a, b = _rrm().gated_scan_backward(g, x, dh, h0, dlast), _rrm().gated_scan_backward(g0, x0, dh, h0, dlast)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    odd = torch.empty(T * n * d + 1, dtype=torch.bfloat16, device="cuda")[1:].view(T, n, d)      # rows on a 2-byte boundary
    odd.copy_(g0)
    c = _rrm().gated_scan(odd, x0, h0)
    close(c[0], _rrm().gated_scan(g0, x0, h0)[0].double(), 2 ** -8 * 5)


def test_streams_captures_and_the_same_bits_again():
    g, x, h0, reset, lens, dh, dlast = _inputs((1500, 2, 64), torch.bfloat16, seed=11)
    fwd = lambda **kw: _rrm().gated_scan(g, x, h0, reset=reset, lengths=lens, **kw)                       # noqa: E731
    bwd = lambda **kw: _rrm().gated_scan_backward(g, x, dh, h0, dlast, reset=reset, lengths=lens, **kw)   # noqa: E731
    first = fwd() + bwd()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = fwd(stream=s) + bwd(stream=s)
    again = fwd() + bwd()                                        # beside the other stream's
    s.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(first, other, again))
    graphs, outs = [], []
    for _ in range(2):                                           # two graphs, each with a workspace of its own
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
    g, x, h0, reset, lens, dh, dlast = _inputs((6, 2, 8), torch.float32)
    for bad in (lambda: rrm.gated_scan(g, x[:5], h0), lambda: rrm.gated_scan(g, x.half(), h0), lambda: rrm.gated_scan(g.double(), x.double()),
                lambda: rrm.gated_scan(g, x, h0[:1]), lambda: rrm.gated_scan(g, x, h0.half()), lambda: rrm.gated_scan(g, x, h0.t().contiguous().t()),
                lambda: rrm.gated_scan(g, x, h0, reset=reset.float()), lambda: rrm.gated_scan(g, x, h0, reset=reset[:3]),
                lambda: rrm.gated_scan(g, x, h0, lengths=lens.long()), lambda: rrm.gated_scan(g.cpu(), x.cpu()),
                lambda: rrm.gated_scan(g[..., ::2], x[..., ::2]), lambda: rrm.gated_scan(g[:1].expand(6, 2, 8), x),
                lambda: rrm.gated_scan(g, x, h=g[:1].expand(6, 2, 8)), lambda: rrm.gated_scan(g[0], x[0]),
                lambda: rrm.gated_scan(g[..., :0], x[..., :0]), lambda: rrm.gated_scan_backward(g, x, dh[:2])):
        with pytest.raises(rrm.RRMError):
            bad()
