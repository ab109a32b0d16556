"""Products of 8-bit integers, bit by bit: sums of integers are exact, and what follows them is the same arithmetic in every
kernel, so results depend neither on how a sum was split nor on which rows a call has beside a row."""
import pytest
import torch

rf = pytest.importorskip("paper_2606_06309_amd.binding")
pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def tensors(rows, K, n, dtype, frames=1):
    g = torch.Generator(device="cuda")
    g.manual_seed(rows + K + n)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(dtype)  # noqa: E731
    whole = lambda *shape: torch.randint(-128, 128, shape, generator=g, device="cuda", dtype=torch.int8)  # noqa: E731
    return dict(x=whole(rows, K), xs=torch.rand(rows, generator=g, device="cuda") * 0.02 + 0.001, w=whole(n, K),
                ws=(torch.rand(n, generator=g, device="cuda") + 0.1) * K ** -0.5 / 40, bias=normal(n), gate=normal(n),
                gates=normal(frames, n), residual=normal(rows, n))


def call(t, act, bias, gate, residual, dtype, workspace=True, rows=None, **kw):
    """The product of t's first rows; workspace False: none is given, whatever the plan would split."""
    x, xs = t["x"][:rows], t["xs"][:rows]
    res = t["residual"][:rows] if residual else None
    b, g = t["bias"] if bias else None, None if gate is None else t[gate]
    if workspace:
        return rf.rf_frame_linear_i8(x, xs, t["w"], t["ws"], b, act, g, res, dtype=dtype, **kw)
    (n_rows, K), n = x.shape, t["w"].shape[0]
    y = torch.empty((n_rows, n), dtype=dtype, device="cuda")
    ids, p = rf._ids([0])
    at = [None if v is None else v.data_ptr() for v in (x, xs, t["w"], t["ws"], b, g, res, y)]
    rf._check(rf.lib.rf_frame_linear_i8(*at, p, 1, 1, n_rows, K, n, rf.ACTIVATIONS[act], 0, rf._dtype_code(dtype), None, 0,
                                        rf._stream(None)))
    return y


EPILOGUES = [(bias, gate, residual) for bias in (False, True) for gate in (None, "gate") for residual in (False, True)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("act", ["none", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("rows,K,n", [(3, 5120, 520), (24, 16384, 264), (40, 8192, 264), (200, 8960, 328), (600, 8960, 512),
                                      (1101, 20480, 1544), (700, 16400, 5128)])
def test_split_and_whole_sums(rows, K, n, act, dtype):
    assert rf.rf_frame_linear_i8_workspace(1, rows, K, n, dtype) > 0
    t = tensors(rows, K, n, dtype)
    for bias, gate, residual in EPILOGUES:
        a = call(t, act, bias, gate, residual, dtype)
        b = call(t, act, bias, gate, residual, dtype, workspace=False)
        assert torch.equal(a, b), (bias, gate, residual, int((a != b).sum()))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("act", ["none", "gelu", "gelu_tanh", "silu"])
def test_rows_alone_and_among_others(act, dtype):
    """The same first rows in the forms of one row to tiles of 256."""
    K, n = 2064, 1544
    t = tensors(9000, K, n, dtype)
    for bias, gate, residual in EPILOGUES:
        most = call(t, act, bias, gate, residual, dtype)
        for rows in (1, 17, 50, 64, 300, 1500, 4000):
            few = call(t, act, bias, gate, residual, dtype, rows=rows)
            assert torch.equal(few, most[:rows]), (rows, bias, gate, residual, int((few != most[:rows]).sum()))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
@pytest.mark.parametrize("N", [7, 100, 743])
def test_frames_and_rows(N, act, dtype):
    """A list of frames, whose gates are their own, against each frame's rows by themselves; compact and at full positions."""
    T, ids, K, n = 9, [0, 2, 3, 8], 1040, 1032
    M = len(ids)
    t = tensors(M * N, K, n, dtype, T)
    pos = (torch.tensor(ids, device="cuda")[:, None] * N + torch.arange(N, device="cuda")).reshape(-1)
    kw = dict(frame_ids=ids, T=T, rows_per_frame=N)
    for residual in (False, True):
        y = call(t, act, True, "gates", residual, dtype, **kw)
        full = torch.zeros((T * N, n), dtype=dtype, device="cuda")
        if residual:
            full[pos] = t["residual"]
        rf.rf_frame_linear_i8(t["x"], t["xs"], t["w"], t["ws"], t["bias"], act, t["gates"], full if residual else None,
                              out=full, out_full=True, **kw)
        assert torch.equal(full[pos], y)
        for i, f in enumerate(ids):
            r = slice(i * N, (i + 1) * N)
            one = rf.rf_frame_linear_i8(t["x"][r], t["xs"][r], t["w"], t["ws"], t["bias"], act, t["gates"][f],
                                        t["residual"][r] if residual else None, dtype=dtype)
            assert torch.equal(one, y[r]), (i, residual, int((one != y[r]).sum()))
