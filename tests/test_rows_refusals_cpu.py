"""What group norm, rows in 8 bits and their products refuse: every wrong argument is turned into an error before any HIP
call (fabricated device addresses, never dereferenced), and the binding turns host tensors, wrong shapes, types and
strides away."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

rf = pytest.importorskip("paper_2606_06309_amd.binding")
lib = rf.lib
INVALID, UNSUPPORTED, RANGE = rf.RF_ERR_INVALID_ARG, rf.RF_ERR_UNSUPPORTED, rf.RF_ERR_RANGE
IN, OUT, GATES, AFFINE = rf.RF_ROWS_IN_FULL, rf.RF_ROWS_OUT_FULL, rf.RF_GATE_PER_FRAME, rf.RF_AFFINE_PER_FRAME


def dev(i):
    return 0x100000000000 + i * 0x10000000000


def _ids(ids):
    return ctypes.cast((ctypes.c_int32 * max(1, len(ids)))(*ids), ctypes.c_void_p)


def quantize(x=dev(0), q=dev(1), s=dev(2), ids=(0, 2), M=None, T=4, N=10, K=64, stride=0, flags=0, dtype=rf.RF_BF16):
    return lib.rf_frame_quantize(x, q, s, None if ids is None else _ids(ids), len(ids or ()) if M is None else M, T, N, K,
                                 stride, flags, dtype, None)


FRAMES = [(dict(ids=()), INVALID), (dict(ids=None, M=2), INVALID), (dict(ids=(2, 0)), INVALID), (dict(ids=(1, 1)), INVALID),
          (dict(ids=(0, 4)), RANGE), (dict(ids=(-1, 0)), RANGE), (dict(T=257), RANGE), (dict(M=5, ids=(0, 1, 2, 3, 4)), RANGE),
          (dict(N=0), INVALID), (dict(N=-1), INVALID), (dict(N=1 << 31), RANGE), (dict(N=1 << 62), RANGE),
          (dict(flags=1 << 9), INVALID), (dict(dtype=2), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED)]


@pytest.mark.parametrize("kw,status", FRAMES + [
    (dict(x=None), INVALID), (dict(q=None), INVALID), (dict(s=None), INVALID), (dict(flags=GATES), INVALID),
    (dict(K=0), INVALID), (dict(K=-16), INVALID), (dict(K=56), UNSUPPORTED), (dict(K=65552), UNSUPPORTED),
    (dict(stride=48), INVALID), (dict(stride=-64), INVALID), (dict(stride=68), UNSUPPORTED), (dict(stride=1 << 60), RANGE),
    (dict(x=dev(0) + 8), UNSUPPORTED), (dict(q=dev(1) + 4), UNSUPPORTED), (dict(s=dev(2) + 2), UNSUPPORTED),
    (dict(q=dev(0)), INVALID), (dict(q=dev(0) + 20 * 64 * 2 - 16), INVALID), (dict(s=dev(0) + 64), INVALID),
    (dict(s=dev(1) + 16), INVALID), (dict(q=dev(0) + 40 * 64 * 2 - 16, flags=IN), INVALID),
    (dict(s=dev(1) + 40 * 64 - 4, flags=OUT), INVALID),
])
def test_quantize(kw, status):
    assert quantize(**kw) == status, lib.rf_last_error()
    assert lib.rf_last_error().decode().startswith("rf_frame_quantize")


def linear(x=dev(0), xs=dev(1), w=dev(2), ws=dev(3), bias=dev(4), gate=dev(5), res=dev(6), y=dev(7), ids=(0, 2), M=None, T=4,
           N=10, K=64, n=32, act=1, flags=0, dtype=rf.RF_BF16, space=None, space_bytes=0):
    return lib.rf_frame_linear_i8(x, xs, w, ws, bias, gate, res, y, None if ids is None else _ids(ids),
                                  len(ids or ()) if M is None else M, T, N, K, n, act, flags, dtype, space, space_bytes, None)


@pytest.mark.parametrize("kw,status", FRAMES + [
    (dict(x=None), INVALID), (dict(xs=None), INVALID), (dict(w=None), INVALID), (dict(ws=None), INVALID), (dict(y=None), INVALID),
    (dict(flags=AFFINE), INVALID), (dict(flags=GATES, gate=None), INVALID), (dict(act=4), INVALID), (dict(act=-1), INVALID),
    (dict(K=0), INVALID), (dict(n=-8), INVALID), (dict(K=72), UNSUPPORTED), (dict(K=65552), UNSUPPORTED),
    (dict(n=36), UNSUPPORTED), (dict(n=34, dtype=rf.RF_F32), UNSUPPORTED),
    (dict(x=dev(0) + 8), UNSUPPORTED), (dict(xs=dev(1) + 1), UNSUPPORTED), (dict(w=dev(2) + 4), UNSUPPORTED),
    (dict(ws=dev(3) + 4), UNSUPPORTED), (dict(bias=dev(4) + 2), UNSUPPORTED), (dict(gate=dev(5) + 8), UNSUPPORTED),
    (dict(res=dev(6) + 8), UNSUPPORTED), (dict(y=dev(7) + 8), UNSUPPORTED),
    (dict(y=dev(0)), INVALID), (dict(y=dev(1) + 64), INVALID), (dict(y=dev(2)), INVALID), (dict(y=dev(3) + 112), INVALID),
    (dict(y=dev(4) + 48), INVALID), (dict(y=dev(5)), INVALID), (dict(y=dev(6) + 64), INVALID),
    (dict(y=dev(5) + 3 * 64, flags=GATES), INVALID), (dict(y=dev(1) + 39 * 4 // 16 * 16, flags=IN), INVALID),
    (dict(space=dev(8), space_bytes=-1), INVALID), (dict(space=dev(8) + 4, space_bytes=64), UNSUPPORTED),
    (dict(space=dev(7), space_bytes=16), INVALID), (dict(space=dev(1) + 64, space_bytes=16), INVALID),
    (dict(space=dev(3) - 16, space_bytes=32), INVALID), (dict(space=dev(0), space_bytes=16), INVALID),
    (dict(N=1 << 29, n=1 << 15, ids=(0,), res=None, y=dev(90)), RANGE),
])
def test_linear(kw, status):
    assert linear(**kw) == status, lib.rf_last_error()
    assert lib.rf_last_error().decode().startswith("rf_frame_linear_i8")


def norm(x=dev(0), w=dev(1), b=dev(2), y=dev(3), ys=None, ids=(0, 2), M=None, T=4, N=10, C=64, G=8, together=1, eps=1e-5, act=1,
         xst=0, yst=0, flags=0, dtype=rf.RF_BF16, space=dev(8), space_bytes=1 << 30):
    return lib.rf_frame_group_norm(x, w, b, y, ys, None if ids is None else _ids(ids), len(ids or ()) if M is None else M, T, N,
                                   C, G, together, eps, act, xst, yst, flags, dtype, space, space_bytes, None)


@pytest.mark.parametrize("kw,status", FRAMES + [
    (dict(x=None), INVALID), (dict(y=None), INVALID), (dict(flags=GATES), INVALID), (dict(flags=AFFINE, w=None, b=None), INVALID),
    (dict(act=4), INVALID), (dict(act=-1), INVALID),
    (dict(eps=0.0), INVALID), (dict(eps=-1e-5), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(eps=1e-31), INVALID), (dict(C=0), INVALID), (dict(G=0), INVALID), (dict(G=-8), INVALID), (dict(G=7), INVALID),
    (dict(G=128), INVALID), (dict(together=0), INVALID), (dict(together=-1), INVALID), (dict(together=3), INVALID),
    (dict(together=4), INVALID), (dict(C=60, G=4), UNSUPPORTED), (dict(C=62, G=2, dtype=rf.RF_F32), UNSUPPORTED),
    (dict(C=8200), UNSUPPORTED), (dict(C=72, ys=dev(4)), UNSUPPORTED), (dict(C=72, ys=dev(4), dtype=rf.RF_F32), UNSUPPORTED),
    (dict(xst=56), INVALID), (dict(yst=-64), INVALID), (dict(xst=68), UNSUPPORTED), (dict(yst=68), UNSUPPORTED),
    (dict(xst=1 << 60), RANGE), (dict(yst=1 << 60), RANGE), (dict(yst=80, ys=dev(4)), INVALID),
    (dict(x=dev(0) + 8), UNSUPPORTED), (dict(w=dev(1) + 2), UNSUPPORTED), (dict(b=dev(2) + 8), UNSUPPORTED),
    (dict(y=dev(3) + 8), UNSUPPORTED), (dict(ys=dev(4) + 2), UNSUPPORTED),
    (dict(y=dev(0) + 128), INVALID), (dict(y=dev(0), yst=128), INVALID), (dict(y=dev(0), flags=OUT), INVALID),
    (dict(y=dev(0), ys=dev(4)), INVALID), (dict(y=dev(0) + 64, xst=128, yst=128, C=64), INVALID),
    (dict(y=dev(1)), INVALID), (dict(y=dev(2) - 16), INVALID), (dict(y=dev(1) + 3 * 128, flags=AFFINE), INVALID),
    (dict(ys=dev(0) + 4), INVALID), (dict(ys=dev(3) + 20 * 64 - 4), INVALID), (dict(ys=dev(1)), INVALID),
    (dict(ys=dev(2) + 124), INVALID),
    (dict(space_bytes=-1), INVALID), (dict(space=dev(8) + 8), UNSUPPORTED), (dict(space=dev(0), space_bytes=16), INVALID),
    (dict(space=dev(3) - 16, space_bytes=32), INVALID), (dict(space=dev(1), space_bytes=16), INVALID),
    (dict(space=dev(2), space_bytes=16), INVALID), (dict(space=dev(4), ys=dev(4), space_bytes=16), INVALID),
])
def test_norm(kw, status):
    assert norm(**kw) == status, lib.rf_last_error()
    assert lib.rf_last_error().decode().startswith("rf_frame_group_norm")


def test_workspace_queries():
    n = ctypes.c_int64(-7)
    ref = ctypes.byref(n)
    assert lib.rf_frame_linear_i8_workspace(1, 9, 64, 64, 0, 256, None) == INVALID
    for args, status in [((0, 9, 64, 64, 0, 256), INVALID), ((1, 0, 64, 64, 0, 256), INVALID), ((1, 9, 72, 64, 0, 256), UNSUPPORTED),
                         ((1, 9, 64, 60, 0, 256), UNSUPPORTED), ((1, 9, 64, 64, 4, 256), UNSUPPORTED),
                         ((256, 1 << 30, 64, 64, 0, 256), RANGE), ((1, 9, 64, 64, 0, 65537), RANGE), ((1, 9, 64, 64, 0, -1), RANGE)]:
        assert lib.rf_frame_linear_i8_workspace(*args, ref) == status
    assert lib.rf_frame_group_norm_workspace(1, 9, 64, 8, 1, 0, 0, 256, None) == INVALID
    for args, status in [((0, 9, 64, 8, 1, 0, 0, 256), INVALID), ((1, 0, 64, 8, 1, 0, 0, 256), INVALID),
                         ((1, 9, 64, 5, 1, 0, 0, 256), INVALID), ((4, 9, 64, 8, 3, 0, 0, 256), INVALID),
                         ((1, 9, 64, 8, 0, 0, 0, 256), INVALID), ((257, 9, 64, 8, 1, 0, 0, 256), RANGE),
                         ((256, 1 << 30, 64, 8, 1, 0, 0, 256), RANGE), ((1, 9, 60, 6, 1, 0, 0, 256), UNSUPPORTED),
                         ((1, 9, 72, 8, 1, 1, 0, 256), UNSUPPORTED), ((1, 9, 8200, 8, 1, 0, 0, 256), UNSUPPORTED),
                         ((1, 9, 64, 8, 1, 0, 3, 256), UNSUPPORTED), ((1, 9, 64, 8, 1, 0, 0, 65537), RANGE)]:
        assert lib.rf_frame_group_norm_workspace(*args, ref) == status
    assert n.value == -7
    for cus in (1, 80, 256, 304, 65536):
        for dtype in (0, 1):
            for rows, K, out in ((1, 16, 8), (1, 65536, 64), (500, 8960, 1536), (2 ** 31 - 1, 16, 8)):
                assert rf.rf_frame_linear_i8_workspace(1, rows, K, out, dtype, cus) >= 0
            for M, N, C, G in ((1, 1, 16, 16), (1, 2 ** 31 - 1, 8192, 8192), (256, 8388607, 16, 1), (6, 1560, 640, 32)):
                for int8 in (False, True):
                    for together in (1, M):
                        assert rf.rf_frame_group_norm_workspace(M, N, C, G, dtype, int8, together, cus) >= 0


def z(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def test_binding_quantize():
    x, i8, f32 = z(12, 64), torch.int8, torch.float32
    ids = dict(frame_ids=np.array([0, 3], dtype=np.int32), T=4, rows_per_frame=6)
    with pytest.raises(ValueError, match="device"):
        rf.rf_frame_quantize(x)
    for kw in (dict(out_full=True), dict(in_full=True), dict(T=2), dict(rows_per_frame=3)):
        with pytest.raises(ValueError, match="frame_ids"):
            rf.rf_frame_quantize(x, **kw)
    with pytest.raises(ValueError, match="must be given"):
        rf.rf_frame_quantize(x, out_full=True, out=z(24, 64, dtype=i8), **ids)
    with pytest.raises(ValueError, match="rows"):
        rf.rf_frame_quantize(x, in_full=True, **ids)
    for kw in (dict(out=z(12, 64)), dict(out=z(12, 48, dtype=i8)), dict(out=z(64, 12, dtype=i8).t()), dict(out_scale=z(12)),
               dict(out_scale=z(11, dtype=f32)), dict(out_scale=z(24, dtype=f32)[::2])):
        with pytest.raises(ValueError):
            rf.rf_frame_quantize(x, **kw)
    for bad in (x[0], z(64, 12).t(), z(1, 64).expand(12, 64)):
        with pytest.raises(ValueError):
            rf.rf_frame_quantize(bad)
    with pytest.raises(TypeError):
        rf.rf_frame_quantize(x.half())


def test_binding_linear():
    x, w, s, t = z(12, 64, dtype=torch.int8), z(32, 64, dtype=torch.int8), z(12, dtype=torch.float32), z(32, dtype=torch.float32)
    with pytest.raises(ValueError, match="device"):
        rf.rf_frame_linear_i8(x, s, w, t)
    with pytest.raises(ValueError, match="activation"):
        rf.rf_frame_linear_i8(x, s, w, t, activation="relu")
    for kw in (dict(bias=z(31)), dict(gate=z(3, 32)), dict(residual=z(12, 31)), dict(out=z(11, 32))):
        with pytest.raises(ValueError):
            rf.rf_frame_linear_i8(x, s, w, t, **kw)
    for args in ((x, t, w, t), (x, s, w, s), (x, s[:, None], w, t), (x, s, w[:, :48], t), (x[0], s, w, t)):
        with pytest.raises(ValueError):
            rf.rf_frame_linear_i8(*args)
    for args in ((x.float(), s, w, t), (x, s.bfloat16(), w, t), (x, s, w.to(torch.uint8), t), (x, s, w, t.double())):
        with pytest.raises(TypeError):
            rf.rf_frame_linear_i8(*args)
    with pytest.raises(TypeError):
        rf.rf_frame_linear_i8(x, s, w, t, bias=z(32), residual=z(12, 32, dtype=torch.float32))
    with pytest.raises(TypeError):
        rf.rf_frame_linear_i8(x, s, w, t, bias=z(32), dtype=torch.float32)
    with pytest.raises(TypeError):
        rf.rf_frame_linear_i8(x, s, w, t, dtype=torch.float16)
    for args in ((z(64, 12, dtype=torch.int8).t(), s, w, t), (x, z(24, dtype=torch.float32)[::2], w, t)):
        with pytest.raises(ValueError, match="contiguous"):
            rf.rf_frame_linear_i8(*args)


def test_binding_norm():
    x = z(12, 64)
    ids = dict(frame_ids=np.array([0, 3], dtype=np.int32), T=4, rows_per_frame=6)
    kw = dict(workspace=None, **ids)
    with pytest.raises(ValueError, match="device"):
        rf.rf_frame_group_norm(x, 8, **kw)
    with pytest.raises(ValueError, match="activation"):
        rf.rf_frame_group_norm(x, 8, activation="relu", **kw)
    for more in (dict(out_full=True), dict(out_full=True, int8=True), dict(in_full=True)):
        with pytest.raises(ValueError):
            rf.rf_frame_group_norm(x, 8, **more, **kw)
    for more in (dict(weight=z(32)), dict(weight=z(4, 64), bias=z(64)), dict(bias=z(3, 64)), dict(out=z(12, 48)),
                 dict(out=z(1, 64).expand(12, 64)), dict(weight=z(128)[::2]), dict(out=z(12, 64, dtype=torch.int8), out_scale=z(12)),
                 dict(out=z(12, 64), int8=True)):
        with pytest.raises(ValueError):
            rf.rf_frame_group_norm(x, 8, **more, **kw)
    with pytest.raises(TypeError):
        rf.rf_frame_group_norm(x, 8, weight=z(64, dtype=torch.float32), **kw)
    with pytest.raises(TypeError):
        rf.rf_frame_group_norm(x, 8, out=z(12, 64, dtype=torch.float32), **kw)
    with pytest.raises(ValueError):
        rf.rf_frame_group_norm(x[0], 8)


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
    both = ((a, "a", torch.bfloat16, True), (None, "none", torch.int8, True), (b, "b", torch.bfloat16, True))
    assert rf._addresses(both) == (0, [a.data_ptr(), None, b.data_ptr()])
    b.index = 1
    with pytest.raises(ValueError, match="b is on cuda:1, the current device is cuda:0"):
        rf._addresses(both)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="a is on cuda:0, the current device is cuda:1"):
        rf._addresses(both)
    with pytest.raises(ValueError, match="c must be a device tensor"):
        rf._addresses(((b, "b", torch.bfloat16, True), (z(3), "c", torch.bfloat16, True)))


def test_constants_match_the_header():
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "rhymeflow.h")) as f:
        text = f.read()
    assert int(re.search(r"#define RF_AFFINE_PER_FRAME (\d+)u", text).group(1)) == rf.RF_AFFINE_PER_FRAME
    for name in ("RF_I8_FEATURES", "RF_NORM_CHANNELS"):
        assert int(re.search(rf"#define {name} (\d+)", text).group(1)) == getattr(rf, name)
