"""Products of 8-bit integers with bias, activation, gate and residual against their definition in 64 bits."""
import pytest
import torch

import block_reference as block
import rows_reference as ref

rf = pytest.importorskip("paper_2606_06309_amd.binding")
pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def draw(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda", dtype=F32) * scale).to(dtype)


def whole(shape, seed, lo=-128):
    """Every int8 value, -128 among them."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randint(lo, 128, shape, generator=g, device="cuda", dtype=torch.int8)


def operands(rows, K, n, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    xs = torch.rand(rows, generator=g, device="cuda") * 0.02 + 0.001
    ws = (torch.rand(n, generator=g, device="cuda") + 0.1) * K ** -0.5 / 40
    return whole((rows, K), seed + 1), xs, whole((n, K), seed + 2), ws


# one row and many, edges of every tile, odd numbers of 16 inputs and of 8 features
SIZES = [(1, 16, 8), (1, 1536, 1536), (2, 48, 40), (6, 1536, 9216), (7, 5120, 5120), (15, 80, 264), (16, 256, 128),
         (17, 272, 136), (24, 10240, 520), (33, 64, 1000), (63, 144, 64), (64, 128, 128), (64, 2048, 2056), (65, 528, 72),
         (100, 5120, 96), (128, 64, 256), (129, 192, 248), (255, 320, 264), (256, 256, 256), (257, 1008, 520),
         (500, 4096, 320), (700, 144, 1544), (1581, 320, 960), (300, 9008, 256), (2100, 64, 2056), (1030, 1040, 1032),
         (5, 65536, 24), (300, 65536, 136)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("size", SIZES)
def test_sizes(size, dtype):
    rows, K, n = size
    xq, xs, wq, ws = operands(rows, K, n, 1)
    block.assert_within(rf.rf_frame_linear_i8(xq, xs, wq, ws, dtype=dtype), *ref.linear_i8(xq, xs, wq, ws, dtype=dtype), f"{size}")
    b, g, r = draw((n,), dtype, 3), draw((n,), dtype, 4), draw((rows, n), dtype, 5)
    y = rf.rf_frame_linear_i8(xq, xs, wq, ws, b, "gelu_tanh", g, r)
    assert y.dtype == dtype
    block.assert_within(y, *ref.linear_i8(xq, xs, wq, ws, b, "gelu_tanh", g, r, dtype), f"{size}")


def test_features_of_four():
    """fp32 rows of a multiple of 4 features."""
    for rows, K, n in [(1, 64, 4), (20, 160, 12), (90, 1040, 260), (500, 320, 1004), (2000, 528, 516)]:
        xq, xs, wq, ws = operands(rows, K, n, 6)
        b, g, r = draw((n,), F32, 3), draw((n,), F32, 4), draw((rows, n), F32, 5)
        y = rf.rf_frame_linear_i8(xq, xs, wq, ws, b, "silu", g, r)
        block.assert_within(y, *ref.linear_i8(xq, xs, wq, ws, b, "silu", g, r, F32), f"{rows} {K} {n}")


@pytest.mark.parametrize("rows,K,n", [(1, 65536, 8), (40, 65536, 136), (600, 65536, 264)])
def test_largest_sums(rows, K, n):
    """-128 x -128 all along the longest row, 2^30, and its negative: exact."""
    xq = torch.full((rows, K), -128, dtype=torch.int8, device="cuda")
    wq = torch.full((n, K), -128, dtype=torch.int8, device="cuda")
    wq[1::2] = 127
    one = torch.ones(rows, device="cuda"), torch.ones(n, device="cuda")
    y = rf.rf_frame_linear_i8(xq, one[0], wq, one[1], dtype=F32)
    assert bool((y[:, 0::2] == 2.0 ** 30).all())
    assert bool((y[:, 1::2] == -128.0 * 127 * K).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("act", ["none", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("rows", [3, 200, 1100])
def test_epilogue(rows, act, dtype):
    K, n = 96, 328
    xq, xs, wq, ws = operands(rows, K, n, 7)
    b, g, r = draw((n,), dtype, 8), draw((n,), dtype, 9), draw((rows, n), dtype, 10)
    ws[:8] *= 40
    for bias in (None, b):
        for gate in (None, g):
            for res in (None, r):
                y = rf.rf_frame_linear_i8(xq, xs, wq, ws, bias, act, gate, res, dtype=dtype)
                block.assert_within(y, *ref.linear_i8(xq, xs, wq, ws, bias, act, gate, res, dtype),
                                    f"{act} {bias is None} {gate is None} {res is None}")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N", [1, 5, 63, 130, 700])
@pytest.mark.parametrize("in_full,out_full", [(False, False), (False, True), (True, False), (True, True)])
def test_frames(N, in_full, out_full, dtype):
    T, ids, K, n = 7, [1, 2, 6], 144, 264
    x, s, w, ws = operands(T * N, K, n, 11)
    b, gate, full = draw((n,), dtype, 13), draw((T, n), dtype, 14), draw((T * N, n), dtype, 15)
    pos = block.positions(ids, N, "cuda")
    listed = torch.zeros(T * N, dtype=torch.bool, device="cuda")
    listed[pos] = True
    s[~listed] = float("nan")
    gate[[0, 3, 4, 5]] = float("nan")
    g = gate[torch.tensor(ids, device="cuda")].repeat_interleave(N, 0)
    want, bound = ref.linear_i8(x[pos], s[pos], w, ws, b, "silu", g, full[pos], dtype)
    xs, ss = (x, s) if in_full else (x[pos], s[pos])
    res = full if out_full else full[pos]
    kw = dict(frame_ids=ids, T=T, rows_per_frame=N, in_full=in_full, out_full=out_full)
    out = draw(res.shape, dtype, 16)
    old = out.clone()
    rf.rf_frame_linear_i8(xs, ss, w, ws, b, "silu", gate, res, out=out, **kw)
    block.assert_within(out[pos] if out_full else out, want, bound)
    if out_full:
        assert torch.equal(out[~listed], old[~listed])
    y = res.clone()      # in place on the residual
    assert rf.rf_frame_linear_i8(xs, ss, w, ws, b, "silu", gate, y, out=y, **kw) is y
    assert torch.equal(y[pos] if out_full else y, out[pos] if out_full else out)
    if out_full:
        assert torch.equal(y[~listed], full[~listed])


@pytest.mark.parametrize("rows", [4, 90, 600])
def test_scales_that_are_not_finite(rows):
    """A scale NaN or infinite spoils its row or its feature and nothing else; scale 0 leaves the bias."""
    K, n = 272, 272
    xq, xs, wq, ws = operands(rows, K, n, 20)
    b = draw((n,), F32, 21)
    want, bound = ref.linear_i8(xq, xs, wq, ws, b)
    xs[2], ws[5], xs[3] = float("nan"), float("inf"), 0.0
    y = rf.rf_frame_linear_i8(xq, xs, wq, ws, b)
    assert bool(torch.isnan(y[2]).all()) and not bool(torch.isfinite(y[:, 5]).any())
    ok = torch.ones((rows, n), dtype=torch.bool, device="cuda")
    ok[2:4], ok[:, 5] = False, False
    block.assert_within(torch.where(ok, y.double(), 0), torch.where(ok, want, 0), torch.where(ok, bound, 0))
    rest = torch.arange(n, device="cuda") != 5
    assert torch.equal(y[3][rest], b[rest])


@pytest.mark.parametrize("rows,K,n", [(3, 5120, 520), (40, 8192, 264), (200, 8960, 328), (600, 8960, 512), (1000, 6144, 1536)])
def test_results_do_not_depend_on_the_workspace(rows, K, n):
    """Sums of integers are the same however they are split."""
    xq, xs, wq, ws = operands(rows, K, n, 22)
    b = draw((n,), BF16, 23)
    need = rf.rf_frame_linear_i8_workspace(1, rows, K, n, BF16)
    with_ws = rf.rf_frame_linear_i8(xq, xs, wq, ws, b, "silu", workspace=torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"))
    without = rf.rf_frame_linear_i8(xq, xs, wq, ws, b, "silu", workspace=torch.empty(16, dtype=torch.uint8, device="cuda")[:0]) \
        if need == 0 else _no_workspace(xq, xs, wq, ws, b)
    assert torch.equal(with_ws, without)


def _no_workspace(xq, xs, wq, ws, b):
    rows, K = xq.shape
    n = wq.shape[0]
    y = torch.empty((rows, n), dtype=BF16, device="cuda")
    ids, p = rf._ids([0])
    rf._check(rf.lib.rf_frame_linear_i8(xq.data_ptr(), xs.data_ptr(), wq.data_ptr(), ws.data_ptr(), b.data_ptr(), None, None,
                                        y.data_ptr(), p, 1, 1, rows, K, n, rf.ACTIVATIONS["silu"], 0, rf.RF_BF16, None, 0,
                                        rf._stream(None)))
    return y


def test_rows_far_apart():
    """Listed frames whose rows are more than 2 GB, and 4 GB, apart."""
    T, N, K, n = 5, 20000, 65536, 72
    ids = [0, 4]
    x = torch.zeros((T * N, K), dtype=torch.int8, device="cuda")
    pos = block.positions(ids, N, "cuda")
    for r in pos.split(4000):
        x[r] = whole((r.numel(), K), int(r[0]) + 1)
    xs = torch.rand(T * N, device="cuda") * 0.01
    wq, ws = whole((n, K), 2), torch.rand(n, device="cuda") * 1e-3
    y = rf.rf_frame_linear_i8(x, xs, wq, ws, frame_ids=ids, T=T, rows_per_frame=N, in_full=True, dtype=F32)
    some = torch.tensor([0, 1, 127, 128, 19999, 20000, 20001, 20100, 39999], device="cuda")
    block.assert_within(y[some], *ref.linear_i8(x[pos[some]], xs[pos[some]], wq, ws))


def test_a_view_at_an_odd_scale():
    """x_scale needs 4 bytes' alignment only."""
    xq, xs, wq, ws = operands(70, 160, 136, 30)
    wide = torch.cat([torch.zeros(1, device="cuda"), xs])
    y = rf.rf_frame_linear_i8(xq, wide[1:], wq, ws, dtype=F32)
    block.assert_within(y, *ref.linear_i8(xq, xs, wq, ws))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("rows", [2, 300])
def test_activations_of_all_arguments(rows, act, dtype):
    """Arguments from -60 to 60, near 0 and large: of the bias, under sums of zero."""
    n, K = 2048, 16
    b = torch.cat([torch.linspace(-60, 60, 1024), torch.linspace(-6, 6, 960), torch.logspace(-30, 30, 64)]).to(dtype).cuda()
    xq, wq = torch.zeros((rows, K), dtype=torch.int8, device="cuda"), torch.zeros((n, K), dtype=torch.int8, device="cuda")
    xs, ws = torch.ones(rows, device="cuda"), torch.ones(n, device="cuda")
    y = rf.rf_frame_linear_i8(xq, xs, wq, ws, b, act)
    block.assert_within(y, *ref.linear_i8(xq, xs, wq, ws, b, act, dtype=dtype))


# tiles of 128 x 128 and of 256 x 256, whole and ragged, with one, two and many frames in a tile
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("K,n", [(2064, 1032), (1040, 2312)])
@pytest.mark.parametrize("M,N", [(1, 5201), (7, 743), (20, 260), (130, 40), (250, 21)])
@pytest.mark.parametrize("full", [False, True])
def test_frames_in_large_tiles(M, N, K, n, full, dtype):
    T = min(M + 3, 256)
    ids = sorted(set(range(T)) - set([0, T // 2, T - 1][:T - M]))
    x, s, w, ws = operands(M * N, K, n, 40)
    b, gate, res = draw((n,), dtype, 41), draw((T, n), dtype, 42), draw((M * N, n), dtype, 43)
    g = gate[torch.tensor(ids, device="cuda")].repeat_interleave(N, 0)
    want, bound = ref.linear_i8(x, s, w, ws, b, "silu", g, res, dtype)
    kw = dict(frame_ids=ids, T=T, rows_per_frame=N)
    if not full:
        block.assert_within(rf.rf_frame_linear_i8(x, s, w, ws, b, "silu", gate, res, **kw), want, bound)
        return
    pos = block.positions(ids, N, "cuda")
    xf, sf = torch.zeros((T * N, K), dtype=torch.int8, device="cuda"), torch.full((T * N,), float("nan"), device="cuda")
    xf[pos], sf[pos] = x, s
    y = draw((T * N, n), dtype, 44)
    y[pos] = res
    old = y.clone()
    rf.rf_frame_linear_i8(xf, sf, w, ws, b, "silu", gate, y, in_full=True, out_full=True, out=y, **kw)
    block.assert_within(y[pos], want, bound)
    listed = torch.zeros(T * N, dtype=torch.bool, device="cuda")
    listed[pos] = True
    assert torch.equal(y[~listed], old[~listed])


@pytest.mark.parametrize("rows,K,n", [(5201, 1040, 2316), (5201, 2064, 1036), (1101, 20480, 1540)])
def test_features_of_four_in_large_tiles(rows, K, n):
    """fp32, with a residual and without; in parts, too."""
    xq, xs, wq, ws = operands(rows, K, n, 45)
    b, g, r = draw((n,), F32, 46), draw((n,), F32, 47), draw((rows, n), F32, 48)
    block.assert_within(rf.rf_frame_linear_i8(xq, xs, wq, ws, b, "gelu", g, r), *ref.linear_i8(xq, xs, wq, ws, b, "gelu", g, r))
    block.assert_within(rf.rf_frame_linear_i8(xq, xs, wq, ws, dtype=F32), *ref.linear_i8(xq, xs, wq, ws))


@pytest.mark.parametrize("rows,K,n", [(1000, 8208, 2056), (1101, 20480, 1544), (5201, 1040, 2312), (700, 16400, 5128)])
def test_large_tiles_do_not_depend_on_the_workspace(rows, K, n):
    xq, xs, wq, ws = operands(rows, K, n, 49)
    b = draw((n,), BF16, 50)
    assert torch.equal(rf.rf_frame_linear_i8(xq, xs, wq, ws, b, "silu"), _no_workspace(xq, xs, wq, ws, b))
