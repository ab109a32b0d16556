"""What a block's operators refuse: every wrong argument is turned into an error before any HIP call (fabricated device
addresses, never dereferenced), and the binding turns host tensors, wrong shapes, types and strides away."""
import ctypes
import math

import numpy as np
import pytest
import torch

rf = pytest.importorskip("paper_2606_06309_amd.binding")
lib = rf.lib
INVALID, UNSUPPORTED, RANGE = rf.RF_ERR_INVALID_ARG, rf.RF_ERR_UNSUPPORTED, rf.RF_ERR_RANGE


def dev(i):
    return 0x100000000000 + i * 0x10000000000


def _idarr(ids):
    return (ctypes.c_int32 * max(1, len(ids)))(*ids)


def rotary(q=dev(0), qo=dev(1), k=dev(2), ko=dev(3), ids=(0, 2), M=None, T=4, H=6, W=5, hq=2, hk=2, d=64,
           dims=(24, 20, 20), theta=(1e4, 1e4, 1e4), origin=(0, 0, 0), step=(1, 1, 1), strides=(0, 0, 0, 0), flags=0,
           dtype=rf.RF_BF16, axes=True):
    ax = rf.rf_rotary_axes()
    ax.dims[:], ax.theta[:], ax.origin[:], ax.step[:] = dims, theta, origin, step
    return lib.rf_rotary(q, qo, k, ko, ctypes.cast(_idarr(ids), ctypes.c_void_p), len(ids) if M is None else M, T, H, W,
                         hq, hk, d, ctypes.byref(ax) if axes else None, *strides, flags, dtype, None)


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), INVALID), (dict(qo=None), INVALID), (dict(ko=None), INVALID), (dict(axes=False), INVALID),
    (dict(ids=()), INVALID), (dict(ids=(2, 0)), INVALID), (dict(ids=(1, 1)), INVALID), (dict(ids=(0, 4)), RANGE),
    (dict(ids=(-1, 0)), RANGE), (dict(T=257), RANGE), (dict(M=5, ids=(0, 1, 2, 3, 4)), RANGE),
    (dict(H=0), INVALID), (dict(W=-3), INVALID), (dict(H=65537), RANGE), (dict(hq=0), INVALID), (dict(hk=0), INVALID),
    (dict(flags=2 << 8), INVALID), (dict(flags=rf.RF_GATE_PER_FRAME), INVALID),
    (dict(dims=(3, 2, 2)), INVALID), (dict(dims=(-2, 4, 4)), INVALID), (dict(dims=(0, 0, 0)), INVALID),
    (dict(dims=(64, 2, 0)), INVALID), (dict(dims=(2 ** 30, 2 ** 30, 2 ** 30)), INVALID),
    (dict(theta=(0.5, 2, 2)), INVALID), (dict(theta=(2, math.inf, 2)), INVALID), (dict(theta=(2, 2, math.nan)), INVALID),
    (dict(origin=(math.nan, 0, 0)), INVALID), (dict(step=(1, math.inf, 1)), INVALID),
    (dict(origin=(2.2e9, 0, 0)), RANGE), (dict(step=(0, 0, -40000.0)), RANGE),
    (dict(d=20, dims=(4, 4, 4)), UNSUPPORTED), (dict(d=264, dims=(4, 4, 4)), UNSUPPORTED),
    (dict(flags=rf.RF_ROTARY_HALVES, dims=(20, 20, 20)), UNSUPPORTED), (dict(dtype=5), UNSUPPORTED),
    (dict(q=dev(0) + 8), UNSUPPORTED), (dict(ko=dev(3) + 4), UNSUPPORTED),
    (dict(strides=(130, 0, 0, 0)), UNSUPPORTED), (dict(strides=(0, 120, 0, 0)), INVALID),
    (dict(strides=(0, 0, -128, 0)), INVALID), (dict(strides=(1 << 60, 0, 0, 0)), RANGE),
    (dict(H=65536, W=65536, ids=(0,), T=256, hq=2 ** 20, hk=2 ** 20), RANGE),
    (dict(qo=dev(0) + 256), INVALID),                        # shifted by a row
    (dict(qo=dev(0), flags=rf.RF_ROWS_OUT_FULL), INVALID),   # in place needs one layout
    (dict(qo=dev(0), strides=(128, 256, 0, 0)), INVALID),    # and one stride
    (dict(qo=dev(2)), INVALID), (dict(ko=dev(1)), INVALID), (dict(ko=dev(1) + 512), INVALID),
    # q_out and k_out in one buffer whose rows are too short for both
    (dict(qo=dev(1), ko=dev(1) + 256, strides=(0, 192, 0, 192)), INVALID),
])
def test_rotary(kw, status):
    assert rotary(**kw) == status, lib.rf_last_error()
    assert lib.rf_last_error().decode().startswith("rf_rotary")


def cross(q=dev(0), k=dev(1), v=dev(2), out=dev(3), lens=None, mask=None, B=2, Lq=9, Lk=7, heads=4, kvh=2, d=64,
          layout=None, dtype=rf.RF_BF16, ws=None, wsb=0):
    lay = None
    if layout is not None:
        plain = dict(q=(Lq * heads * d, heads * d, d), k=(Lk * kvh * d, kvh * d, d), v=(Lk * kvh * d, kvh * d, d),
                     out=(Lq * heads * d, heads * d, d))
        lay = rf.rf_cross_layout()
        for n, s in {**plain, **layout}.items():
            getattr(lay, n)[:] = s
        lay = ctypes.byref(lay)
    return lib.rf_cross_attention(q, k, v, out, lens, mask, B, Lq, Lk, heads, kvh, d, lay, dtype, ws, wsb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(out=None), INVALID),
    (dict(B=0), INVALID), (dict(Lq=0), INVALID), (dict(Lk=0), INVALID), (dict(Lk=-4), INVALID), (dict(heads=0), INVALID),
    (dict(kvh=0), INVALID), (dict(kvh=3), INVALID), (dict(heads=2, kvh=4), INVALID), (dict(d=32), UNSUPPORTED),
    (dict(d=96), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED), (dict(q=dev(0) + 2), UNSUPPORTED),
    (dict(out=dev(3) + 8), UNSUPPORTED), (dict(lens=dev(4) + 2), UNSUPPORTED),
    (dict(B=2 ** 30, Lq=2 ** 30, heads=64, kvh=64), RANGE), (dict(B=2 ** 16, Lq=2 ** 14, heads=8, kvh=8), RANGE),
    (dict(Lk=2 ** 30 + 1), RANGE), (dict(layout=dict(k=(0, 56, 64))), INVALID), (dict(layout=dict(v=(0, 0, 64))), INVALID),
    (dict(out=dev(0)), INVALID), (dict(out=dev(1) + 64), INVALID), (dict(out=dev(2) - 256), INVALID),
    (dict(out=dev(3), lens=dev(3) + 16), INVALID), (dict(out=dev(3), mask=dev(3) + 5), INVALID),
    (dict(layout=dict(q=(-64, 256, 64))), INVALID), (dict(layout=dict(k=(0, 132, 64))), UNSUPPORTED),
    (dict(layout=dict(v=(0, 1 << 23, 64))), UNSUPPORTED), (dict(layout=dict(q=(1 << 62, 256, 64))), RANGE),
    (dict(layout=dict(q=(1 << 59, 256, 64)), B=2 ** 10), RANGE),
    (dict(layout=dict(out=(0, 256, 64))), INVALID), (dict(layout=dict(out=(9 * 256, 256, 56))), INVALID),
    (dict(layout=dict(out=(8 * 256, 256, 64))), INVALID),
    (dict(ws=dev(5), wsb=-1), INVALID), (dict(ws=dev(5) + 4, wsb=64), UNSUPPORTED), (dict(ws=dev(3), wsb=64), INVALID),
    (dict(ws=dev(0) + 1024, wsb=64), INVALID),
])
def test_cross(kw, status):
    assert cross(**kw) == status, lib.rf_last_error()
    assert lib.rf_last_error().decode().startswith("rf_cross_attention")


def linear(x=dev(0), w=dev(1), b=dev(2), g=dev(3), r=dev(4), y=dev(5), ids=(0, 2), M=None, T=4, N=10, K=64, n=32, act=0,
           flags=0, dtype=rf.RF_BF16, ws=None, wsb=0):
    return lib.rf_frame_linear(x, w, b, g, r, y, ctypes.cast(_idarr(ids), ctypes.c_void_p),
                               len(ids) if M is None else M, T, N, K, n, act, flags, dtype, ws, wsb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(y=None), INVALID), (dict(N=0), INVALID), (dict(K=0), INVALID),
    (dict(n=-8), INVALID), (dict(ids=()), INVALID), (dict(ids=(2, 1)), INVALID), (dict(ids=(0, 4)), RANGE),
    (dict(T=300), RANGE), (dict(flags=8), INVALID), (dict(flags=rf.RF_ROTARY_HALVES), INVALID),
    (dict(g=None, flags=rf.RF_GATE_PER_FRAME), INVALID), (dict(act=4), INVALID), (dict(act=-1), INVALID),
    (dict(dtype=3), UNSUPPORTED), (dict(K=60), UNSUPPORTED), (dict(n=36), UNSUPPORTED),
    (dict(K=62, dtype=rf.RF_F32), UNSUPPORTED), (dict(K=1 << 22), UNSUPPORTED),
    (dict(K=1 << 21, dtype=rf.RF_F32), UNSUPPORTED), (dict(N=1 << 31), RANGE),
    (dict(N=(1 << 31) - 1, ids=(0,), T=256, K=(1 << 21) - 8, n=2 ** 31 - 8), RANGE),
    (dict(b=dev(2) + 2), UNSUPPORTED), (dict(x=dev(0) + 8), UNSUPPORTED),
    (dict(y=dev(0)), INVALID), (dict(y=dev(1) + 128), INVALID), (dict(y=dev(2)), INVALID), (dict(y=dev(3)), INVALID),
    (dict(y=dev(4) + 64), INVALID), (dict(y=dev(3) + 192, flags=rf.RF_GATE_PER_FRAME), INVALID),
    (dict(ws=dev(6), wsb=-5), INVALID), (dict(ws=dev(6) + 8, wsb=16), UNSUPPORTED), (dict(ws=dev(1), wsb=16), INVALID),
    (dict(ws=dev(5) + 16, wsb=16), INVALID),
])
def test_linear(kw, status):
    assert linear(**kw) == status, lib.rf_last_error()
    assert lib.rf_last_error().decode().startswith("rf_frame_linear")


def test_workspace_queries():
    n = ctypes.c_int64(-7)
    ref = ctypes.byref(n)
    assert lib.rf_cross_attention_workspace(1, 1, 9, 2, 1, 64, 0, 256, None) == INVALID
    for args, status in [((0, 1, 9, 2, 1, 64, 0, 256), INVALID), ((1, 1, 9, 2, 4, 64, 0, 256), INVALID),
                         ((1, 1, 9, 2, 1, 80, 0, 256), UNSUPPORTED), ((1, 1, 9, 2, 1, 64, 9, 256), UNSUPPORTED),
                         ((1, 1, 9, 2, 1, 64, 0, -1), RANGE), ((1, 1, 9, 2, 1, 64, 0, 70000), RANGE)]:
        assert lib.rf_cross_attention_workspace(*args, ref) == status
    assert lib.rf_frame_linear_workspace(1, 9, 64, 64, 0, 256, None) == INVALID
    for args, status in [((0, 9, 64, 64, 0, 256), INVALID), ((1, 0, 64, 64, 0, 256), INVALID),
                         ((1, 9, 60, 64, 0, 256), UNSUPPORTED), ((1, 9, 64, 64, 4, 256), UNSUPPORTED),
                         ((256, 1 << 30, 64, 64, 0, 256), RANGE), ((1, 9, 64, 64, 0, 65537), RANGE)]:
        assert lib.rf_frame_linear_workspace(*args, ref) == status
    assert n.value == -7
    for cus in (1, 80, 256, 304):
        for dtype in (0, 1):
            for Lq, Lk in ((1, 1), (1, 10 ** 6), (64, 5000), (100000, 512)):
                assert rf.rf_cross_attention_workspace(2, Lq, Lk, 4, 2, 64, dtype, cus) >= 0
            for rows, K, out in ((1, 8, 8), (1, 20480, 64), (500, 8960, 1536), (2 ** 31 - 1, 8, 8)):
                assert rf.rf_frame_linear_workspace(1, rows, K, out, dtype, cus) >= 0


def z(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def test_binding_rotary():
    x = z(12, 2, 64)
    kw = dict(frame_ids=[0, 2], T=4, H=2, W=3, dims=(24, 20, 20))
    with pytest.raises(ValueError, match="device"):
        rf.rf_rotary(x, out=z(12, 2, 64), **kw)
    with pytest.raises(ValueError, match="rows"):
        rf.rf_rotary(x, out=z(12, 2, 64), in_full=True, **kw)
    with pytest.raises(ValueError, match="out must be given"):
        rf.rf_rotary(x, out_full=True, **kw)
    with pytest.raises(ValueError, match="contiguous"):
        rf.rf_rotary(z(12, 64, 2).transpose(1, 2), out=z(12, 2, 64), **kw)
    with pytest.raises(ValueError, match="rows overlap"):
        rf.rf_rotary(z(1, 2, 64).expand(12, 2, 64), out=z(12, 2, 64), **kw)
    with pytest.raises(TypeError):
        rf.rf_rotary(x, out=z(12, 2, 64, dtype=torch.float32), **kw)
    with pytest.raises(TypeError):
        rf.rf_rotary(x.half(), out=x.half(), **kw)
    with pytest.raises(ValueError):
        rf.rf_rotary(x, k=z(12, 2, 32), out=z(12, 2, 64), k_out=z(12, 2, 32), **kw)
    with pytest.raises(ValueError):
        rf.rf_rotary(x[0], **kw)


def test_binding_cross():
    q, k = z(2, 5, 4, 64), z(2, 7, 2, 64)
    with pytest.raises(ValueError, match="device"):
        rf.rf_cross_attention(q, k, k)
    for bad in ((q, k, z(2, 6, 2, 64)), (q, z(1, 7, 2, 64), z(1, 7, 2, 64)), (q, z(2, 7, 2, 32), z(2, 7, 2, 32)),
                (q[0], k, k)):
        with pytest.raises(ValueError):
            rf.rf_cross_attention(*bad)
    with pytest.raises(ValueError, match="contiguous"):
        rf.rf_cross_attention(q, z(2, 7, 64, 2).transpose(2, 3), k)
    with pytest.raises(ValueError, match="q's shape"):
        rf.rf_cross_attention(q, k, k, out=z(2, 5, 4, 32))
    for lens in (torch.zeros(2, dtype=torch.int64), torch.zeros(3, dtype=torch.int32),
                 torch.zeros(4, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError, match="kv_lengths"):
            rf.rf_cross_attention(q, k, k, lens)
    for mask in (torch.zeros((2, 7)), torch.zeros((1, 7), dtype=torch.bool), torch.zeros((7, 2), dtype=torch.bool).t()):
        with pytest.raises(ValueError, match="key_mask"):
            rf.rf_cross_attention(q, k, k, key_mask=mask)
    with pytest.raises(TypeError):
        rf.rf_cross_attention(q, k, k.float())


def test_binding_linear():
    x, w = z(12, 64), z(32, 64)
    with pytest.raises(ValueError, match="device"):
        rf.rf_frame_linear(x, w)
    with pytest.raises(ValueError, match="activation"):
        rf.rf_frame_linear(x, w, activation="relu")
    with pytest.raises(ValueError, match="frame_ids"):
        rf.rf_frame_linear(x, w, out_full=True)
    with pytest.raises(ValueError, match="rows_per_frame"):
        rf.rf_frame_linear(x, w, frame_ids=[0], T=2)
    ids = dict(frame_ids=np.array([0, 3], dtype=np.int32), T=4, rows_per_frame=6)
    with pytest.raises(ValueError, match="out must be given"):
        rf.rf_frame_linear(x, w, out_full=True, **ids)
    for kw in (dict(bias=z(31)), dict(gate=z(3, 32)), dict(residual=z(12, 31)), dict(out=z(11, 32)),
               dict(residual=z(12, 32), out=z(24, 32), out_full=True), dict(in_full=True)):
        with pytest.raises(ValueError):
            rf.rf_frame_linear(x, w, **kw, **ids)
    for kw in (dict(bias=z(64)[::2]), dict(residual=z(32, 12).t())):
        with pytest.raises(ValueError, match="contiguous"):
            rf.rf_frame_linear(x, w, **kw)
    with pytest.raises(TypeError):
        rf.rf_frame_linear(x, w, bias=z(32, dtype=torch.float32))
    with pytest.raises(ValueError):
        rf.rf_frame_linear(x, z(32, 56))



def test_tensors_of_another_device_are_refused(monkeypatch):
    class Fake(torch.Tensor):
        is_cuda = True
        index = 0

        def get_device(self):
            return self.index

        @property
        def device(self):
            return torch.device("cuda", self.index)
    a, b = z(4, 8).as_subclass(Fake), z(4, 8).as_subclass(Fake)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    assert rf._on_device(((a, "a"), (None, "none"), (b, "b")))[0] == 0
    b.index = 1
    with pytest.raises(ValueError, match="cuda:1"):
        rf._on_device(((a, "a"), (b, "b")))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device is cuda:1"):
        rf._on_device(((a, "a"),))


def test_constants_match_the_header():
    import os
    import re
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "rhymeflow.h")) as f:
        text = f.read()
    for name in ("RF_ROWS_IN_FULL", "RF_ROWS_OUT_FULL", "RF_GATE_PER_FRAME", "RF_ROTARY_HALVES", "RF_ROTARY_INVERSE"):
        assert int(re.search(rf"#define {name} (\d+)u", text).group(1)) == getattr(rf, name)
    for name, code in rf.ACTIVATIONS.items():
        assert int(re.search(rf"#define RF_ACT_{name.upper()} (\d+)", text).group(1)) == code
