"""The head operators' argument checks, which come before any device work: the calls return their status on a machine without
a GPU too (pointers are dummies that are never dereferenced)."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, SHAPE, DTYPE, CAPACITY, UNSUPPORTED = -1, -2, -3, -5, -8
F32, I8, BF16, F16 = 0, 1, 3, 4
P = ctypes.c_void_p(4096)
ODD = ctypes.c_void_p(4097)


def _rrm():
    import paper_1802_09723_b200 as rrm
    return rrm


def _make(cls, base, kw):
    d = cls()
    for k, v in {**base, **kw}.items():
        setattr(d, k, v)
    return d


def _norm(**kw):
    return _make(_rrm().NormDesc, dict(dtype=F32, act=0, n=2, pixels=9, c=16, groups=4, eps=1e-5), kw)


def _ff(**kw):
    return _make(_rrm().FfDesc, dict(dtype=BF16, act=5, m=4, k=32, f=24), kw)


def _scan(**kw):
    return _make(_rrm().ScanDesc, dict(dtype=F32, frames=5, n=2, d=8), kw)


def test_the_structs_mirror_the_header():
    rrm = _rrm()
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "rrm.h")).read(), flags=re.S)
    for name, cls in (("rrm_norm_desc", rrm.NormDesc), ("rrm_ff_desc", rrm.FfDesc), ("rrm_scan_desc", rrm.ScanDesc)):
        body = re.search(r"typedef struct \{([^}]*)\}\s*" + name, text).group(1)
        fields = []
        for line in body.split(";"):
            m = re.match(r"\s*(int32_t|int64_t|float)\s+(.*)", line.strip(), flags=re.S)
            if m:
                fields += [(f.strip(), m.group(1)) for f in m.group(2).split(",")]
        kind = {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float}
        assert [(n, kind[t]) for n, t in fields] == list(cls._fields_), name


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=I8), DTYPE), (dict(dtype=2), DTYPE), (dict(dtype=9), DTYPE), (dict(act=2), INVALID), (dict(act=7), INVALID), (dict(act=-1), INVALID),
    (dict(eps=0.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(reserved=1), INVALID), (dict(n=-1), SHAPE), (dict(pixels=-1), SHAPE),
    (dict(c=0), SHAPE), (dict(groups=0), SHAPE), (dict(groups=5), SHAPE), (dict(c=131072, groups=65536), CAPACITY),
    (dict(c=8192, groups=1), CAPACITY), (dict(pixels=(1 << 30) + 1), CAPACITY), (dict(x_pixel=-16), SHAPE), (dict(y_pixel=8), SHAPE),
    (dict(y_image=16), SHAPE)])
def test_norm_descriptions(kw, want):
    L = _rrm().lib()
    d = _norm(**kw)
    assert L.rrm_group_norm_workspace(ctypes.byref(d), 0) == want
    assert L.rrm_group_norm(ctypes.byref(d), P, P, P, P, P, P, 1 << 40, None) == want


def test_norm_pointers_and_workspaces():
    L = _rrm().lib()
    d = _norm()
    ref = ctypes.byref(d)
    assert L.rrm_group_norm(None, P, P, P, P, P, P, 1 << 20, None) == INVALID
    assert L.rrm_group_norm_workspace(None, 0) == INVALID
    need = L.rrm_group_norm_workspace(ref, 0)
    assert need > 0
    assert L.rrm_group_norm(ref, P, P, P, P, P, P, 0, None) == CAPACITY
    assert L.rrm_group_norm(ref, P, P, P, P, P, None, need, None) == INVALID
    assert L.rrm_group_norm(ref, P, P, P, P, P, ctypes.c_void_p(4096 + 16), need, None) == INVALID
    for i in (0, 1, 2, 3, 4):
        args = [P] * 5
        args[i] = ODD
        assert L.rrm_group_norm(ref, *args, P, need, None) == INVALID
    for i in (0, 3):
        args = [P] * 5
        args[i] = None
        assert L.rrm_group_norm(ref, *args, P, need, None) == INVALID
    back = L.rrm_group_norm_workspace(ref, 1)
    assert back >= 2 * 16 * 2 * 4
    assert L.rrm_group_norm_backward(ref, P, P, P, P, None, P, P, P, P, back, None) == INVALID          # no statistics
    assert L.rrm_group_norm_backward(ref, P, P, P, P, ctypes.c_void_p(4100), P, P, P, P, back, None) == INVALID
    assert L.rrm_group_norm_backward(ref, P, P, P, P, P, P, P, P, P, 16, None) == CAPACITY
    small = _norm(dx_pixel=8)
    assert L.rrm_group_norm_backward(ctypes.byref(small), P, P, P, P, P, P, P, P, P, 1 << 40, None) == SHAPE
    assert L.rrm_group_norm(ctypes.byref(_norm(n=0)), None, None, None, None, None, None, 0, None) == 0    # nothing to do
    assert L.rrm_net_group_norm(None, 0, 1, ctypes.c_float(1e-5), 0, P, P, P, P, P, 0, None) == INVALID
    assert L.rrm_net_group_norm_workspace(None, 0, 1) == INVALID


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=F16), DTYPE), (dict(dtype=I8), DTYPE), (dict(act=2), INVALID), (dict(act=9), INVALID), (dict(unaligned=2), INVALID),
    (dict(reserved=1), INVALID), (dict(m=-1), SHAPE), (dict(k=0), SHAPE), (dict(f=0), SHAPE), (dict(m=(1 << 24) + 1), CAPACITY), (dict(k=(1 << 20) + 1), CAPACITY),
    (dict(f=(1 << 20) + 1), CAPACITY), (dict(ld_x=31), SHAPE), (dict(ld_w=31), SHAPE), (dict(ld_y=23), SHAPE), (dict(ld_x=1 << 40), CAPACITY)])
def test_ff_descriptions(kw, want):
    L = _rrm().lib()
    d = _ff(**kw)
    assert L.rrm_gated_ff_workspace(ctypes.byref(d), 0) == want
    assert L.rrm_gated_ff(ctypes.byref(d), P, P, P, P, P, P, P, 1 << 40, None) == want


def test_ff_pointers_and_workspaces():
    L = _rrm().lib()
    d = _ff()
    ref = ctypes.byref(d)
    assert L.rrm_gated_ff(None, P, P, P, P, P, P, P, 0, None) == INVALID
    assert L.rrm_gated_ff_workspace(ref, 0) == 0                     # 16-byte rows of bf16 are taken where they lie
    assert L.rrm_gated_ff_workspace(ctypes.byref(_ff(k=33)), 0) > 0
    assert L.rrm_gated_ff_workspace(ctypes.byref(_ff(unaligned=1)), 0) > 0
    for i in (0, 1, 2, 5):
        args = [P] * 6
        args[i] = None
        assert L.rrm_gated_ff(ref, *args, P, 0, None) == INVALID
    for i in range(6):
        args = [P] * 6
        args[i] = ODD
        assert L.rrm_gated_ff(ref, *args, P, 0, None) == INVALID
    assert L.rrm_gated_ff(ref, ctypes.c_void_p(4104), P, P, P, P, P, P, 0, None) == INVALID              # not 16-byte aligned, not said to be loose
    assert L.rrm_gated_ff(ctypes.byref(_ff(k=33)), P, P, P, P, P, P, P, 16, None) == CAPACITY
    need = L.rrm_gated_ff_workspace(ref, 1)
    assert need > 0
    back = lambda *a, ws=P, n=need: L.rrm_gated_ff_backward(ref, P, P, P, P, P, P, *a, ws, n, None)      # noqa: E731
    assert back(P, P, None, P, P) == INVALID and back(P, None, P, P, P) == INVALID                       # one of a pair
    assert back(P, P, P, P, P, n=8) == CAPACITY and back(P, P, P, P, P, ws=None) == INVALID
    assert back(ODD, P, P, P, P) == INVALID and back(P, P, P, ODD, P) == INVALID
    assert L.rrm_gated_ff_backward(ctypes.byref(_ff(ld_dw=16)), P, P, P, P, P, P, P, P, P, P, P, P, 1 << 40, None) == SHAPE
    assert L.rrm_gated_ff(ctypes.byref(_ff(m=0)), None, None, None, None, None, None, None, 0, None) == 0


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=I8), DTYPE), (dict(fill=2), INVALID), (dict(reserved=3), INVALID), (dict(frames=-1), SHAPE), (dict(n=0), SHAPE), (dict(d=0), SHAPE),
    (dict(frames=(1 << 30) + 1), CAPACITY), (dict(n=1 << 20, d=1 << 20), CAPACITY), (dict(frames=1 << 20, n=1 << 20, d=1), CAPACITY),
    (dict(g_frame=-1), SHAPE), (dict(h_stream=4), SHAPE), (dict(h_frame=8), SHAPE)])
def test_scan_descriptions(kw, want):
    L = _rrm().lib()
    d = _scan(**kw)
    assert L.rrm_gated_scan_workspace(ctypes.byref(d), 0) == want
    assert L.rrm_gated_scan(ctypes.byref(d), P, P, P, P, P, P, P, P, 1 << 50, None) == want


def test_scan_pointers_and_workspaces():
    L = _rrm().lib()
    d = _scan()
    ref = ctypes.byref(d)
    assert L.rrm_gated_scan(None, P, P, P, P, P, P, P, P, 0, None) == INVALID
    assert L.rrm_gated_scan_workspace(ref, 0) == 0
    for i in (0, 1, 5):
        args = [P] * 7
        args[i] = None
        assert L.rrm_gated_scan(ref, *args, P, 0, None) == INVALID
    for i in (0, 1, 2, 4, 5, 6):                                     # (a reset is bytes)
        args = [P] * 7
        args[i] = ODD
        assert L.rrm_gated_scan(ref, *args, P, 0, None) == INVALID
    long = _scan(frames=5000)
    need = L.rrm_gated_scan_workspace(ctypes.byref(long), 1)
    assert need > L.rrm_gated_scan_workspace(ctypes.byref(long), 0) > 0
    assert L.rrm_gated_scan(ctypes.byref(long), P, P, P, P, P, P, P, P, 16, None) == CAPACITY
    assert L.rrm_gated_scan(ctypes.byref(long), P, P, P, P, P, P, P, None, need, None) == INVALID
    assert L.rrm_gated_scan_backward(ref, P, P, P, P, P, P, P, None, P, P, P, 0, None) == INVALID        # dg missing
    assert L.rrm_gated_scan_backward(ctypes.byref(_scan(dx_stream=4)), P, P, P, P, P, P, P, P, P, P, P, 1 << 40, None) == SHAPE


def test_layers_do_not_take_the_head_s_types_and_activations():
    rrm = _rrm()
    L = rrm.lib()
    base = dict(kind=0, dtype=0, n=1, c_in=4, h=8, w=8, c_out=4, kh=3, kw=3, stride=1, pad=1, shift=-1, res=-1)
    for kw, want in ((dict(dtype=BF16), DTYPE), (dict(dtype=F16), DTYPE), (dict(act=4), INVALID), (dict(act=5), INVALID), (dict(act=6), INVALID)):
        h = ctypes.c_void_p()
        d = _make(rrm.LayerDesc, base, kw)
        assert L.rrm_layer_create(ctypes.byref(h), ctypes.byref(d), P, None) == want and not h.value

