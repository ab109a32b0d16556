"""What rf_rotary passes on as its axes: the values at the time of the call, whatever kind of numbers they come as. The
library's entry is replaced by one that keeps them; no GPU is used."""
import ctypes

import numpy as np
import pytest
import torch

rf = pytest.importorskip("paper_2606_06309_amd.binding")


class Library:
    def rf_rotary(self, *args):
        axes = ctypes.cast(args[12], ctypes.POINTER(rf.rf_rotary_axes)).contents
        self.axes = {name: list(getattr(axes, name)) for name in ("dims", "theta", "origin", "step")}
        return rf.RF_OK


@pytest.fixture
def axes_of(monkeypatch):
    library = Library()
    monkeypatch.setattr(rf, "lib", library)
    monkeypatch.setattr(rf, "_on_device", lambda tensors: (0, [1] * len(tensors)))
    x, out = torch.zeros((12, 2, 64), dtype=torch.bfloat16), torch.zeros((12, 2, 64), dtype=torch.bfloat16)

    def call(dims=(24, 20, 20), **kw):
        rf.rf_rotary(x, [0, 2], 4, 2, 3, dims, out=out, stream=0, **kw)
        return library.axes
    return call


def test_values_of_the_call(axes_of):
    want = dict(dims=[24, 20, 20], theta=[100.0, 2.5, 1e4], origin=[0.5, -3.0, 7.0], step=[1.0, 0.25, 2.0])
    for kind in (tuple, list, np.array, torch.tensor):
        assert axes_of(kind([24, 20, 20]), theta=kind([100.0, 2.5, 1e4]), origin=kind([0.5, -3.0, 7.0]),
                       step=kind([1.0, 0.25, 2.0])) == want, kind
    assert axes_of((24.0, 20.0, 20.0))["dims"] == [24, 20, 20]
    for theta in (50, 50.0, np.float32(50), np.float64(50), torch.tensor(50.0), (50, 50, 50)):
        assert axes_of(theta=theta)["theta"] == [50.0] * 3


@pytest.mark.parametrize("name", ["origin", "step", "theta"])
@pytest.mark.parametrize("kind", [tuple, list])
def test_numbers_that_change_between_calls(axes_of, name, kind):
    """A window that moves: one of the three is a tensor that the caller counts up in place."""
    moving = torch.tensor(2.0, dtype=torch.float64)
    values = kind([moving, 3.0, 4.0])
    for i in range(3):
        assert axes_of(**{name: values})[name] == [2.0 + i, 3.0, 4.0]
        moving += 1


def test_dims_that_change_between_calls(axes_of):
    n = torch.tensor(20)
    assert axes_of([24, n, 20])["dims"] == [24, 20, 20]
    n -= 4
    assert axes_of([24, n, 20])["dims"] == [24, 16, 20]


def test_refusals(axes_of):
    for dims in ((24.5, 20, 20), (24, 20, float("nan")), np.array([24, 20, 19.9]), torch.tensor([24, 20, 20.5])):
        with pytest.raises(ValueError):
            axes_of(dims)
    for kw in (dict(dims=(24, 20)), dict(origin=(0.0, 0.0)), dict(step=(1.0,) * 4), dict(theta=(2.0, 3.0))):
        with pytest.raises(ValueError):
            axes_of(**kw)
