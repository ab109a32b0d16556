"""Rotary positions against their definition in 64 bits."""
import numpy as np
import pytest
import torch

import block_reference as ref

rf = pytest.importorskip("paper_2606_06309_amd.binding")
pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def draw(shape, dtype, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda", dtype=F32).to(dtype)


# T, H, W, listed frames, q heads, k heads, head_dim, dims
SHAPES = [
    (1, 1, 1, [0], 1, 1, 8, (2, 0, 0)),
    (1, 1, 1, [0], 3, 1, 64, (16, 24, 24)),
    (5, 8, 8, [0, 2, 4], 2, 2, 64, (24, 20, 20)),
    (7, 3, 5, [1, 6], 5, 1, 128, (44, 42, 42)),
    (3, 17, 31, [2], 4, 2, 80, (28, 26, 26)),
    (4, 9, 7, [0, 1, 2, 3], 3, 3, 128, (0, 10, 12)),
    (2, 5, 33, [1], 1, 4, 256, (80, 88, 88)),
    (1, 37, 53, [0], 2, 1, 64, (0, 32, 32)),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("in_full,out_full", [(False, False), (False, True), (True, False), (True, True)])
def test_rotary(shape, dtype, in_full, out_full):
    T, H, W, ids, hq, hk, d, dims = shape
    N = H * W
    pos = ref.positions(ids, N, "cuda")
    q, k = draw((T * N, hq, d), dtype, 1), draw((T * N, hk, d), dtype, 2)
    qc, kc = q[pos], k[pos]
    rows = T * N if out_full else len(ids) * N
    qo, ko = draw((rows, hq, d), dtype, 3), draw((rows, hk, d), dtype, 4)
    q0, k0 = qo.clone(), ko.clone()
    rf.rf_rotary(q if in_full else qc, ids, T, H, W, dims, k=k if in_full else kc, out=qo, k_out=ko, in_full=in_full,
                 out_full=out_full)
    for x, y, old in ((qc, qo, q0), (kc, ko, k0)):
        want, bound = ref.rotary(x, ids, H, W, dims)
        ref.assert_within(y[pos] if out_full else y, want, bound, f"{shape}")
        if out_full:
            other = torch.ones(rows, dtype=torch.bool, device="cuda")
            other[pos] = False
            assert torch.equal(y[other], old[other])
        R = sum(dims)
        assert torch.equal((y[pos] if out_full else y)[..., R:], x[..., R:])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,dims", [(64, (16, 24, 24)), (128, (16, 24, 24)), (64, (0, 32, 32)), (80, (2, 30, 32)),
                                    (16, (4, 6, 6)), (256, (0, 16, 0))])
def test_halves(d, dims, dtype):
    T, H, W, ids = 6, 5, 9, [0, 3, 5]
    x, k = draw((len(ids) * H * W, 3, d), dtype, 5), draw((len(ids) * H * W, 2, d), dtype, 6)
    y, yk = rf.rf_rotary(x, ids, T, H, W, dims, k=k, halves=True)
    for a, b in ((x, y), (k, yk)):
        want, bound = ref.rotary(a, ids, H, W, dims, halves=True)
        ref.assert_within(b, want, bound)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_far_and_fractional_positions(dtype):
    """Angles of positions near 2^31 turns and of steps that do not divide."""
    T, H, W, ids, dims = 4, 6, 6, [1, 3], (8, 28, 28)
    kw = dict(theta=(100.0, 10000.0, 1.0), origin=(2.0e9, -3.0e5, 0.25), step=(1.0, 0.37, -113.0))
    x = draw((len(ids) * H * W, 2, 64), dtype, 7)
    y = rf.rf_rotary(x, ids, T, H, W, dims, **kw)
    want, bound = ref.rotary(x, ids, H, W, dims, **kw)
    # the reference's own angle is rounded at 2^-53 of up to 2^31 radians, as is the kernel's, in turns
    slack = 4 * 2.0e9 * 2.0 ** -53 * (x.double().abs().amax(-1, keepdim=True) * 2)
    ref.assert_within(y, want, bound + slack)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("halves", [False, True])
def test_inverse_is_the_transpose(halves, dtype):
    """<g, rot(x)> = <rot^-1(g), x>: the inverse takes gradients back; and it undoes the rotation."""
    T, H, W, ids, dims = 5, 4, 7, [0, 4], (16, 24, 24)
    x, g = draw((2 * H * W, 3, 72), dtype, 8), draw((2 * H * W, 3, 72), dtype, 9)
    gx = rf.rf_rotary(g, ids, T, H, W, dims, halves=halves, inverse=True)
    want, bound = ref.rotary(g, ids, H, W, dims, halves=halves, inverse=True)
    ref.assert_within(gx, want, bound)
    fwd, _ = ref.rotary(x, ids, H, W, dims, halves=halves)
    lhs, rhs = (g.double() * fwd).sum(), (want * x.double()).sum()
    assert abs(float(lhs - rhs)) <= 1e-10 * float((g.double() * fwd).abs().sum())
    y = rf.rf_rotary(x, ids, T, H, W, dims, halves=halves)
    back = rf.rf_rotary(y, ids, T, H, W, dims, halves=halves, inverse=True)
    _, b1 = ref.rotary(x, ids, H, W, dims, halves=halves)
    _, b2 = ref.rotary(y, ids, H, W, dims, halves=halves, inverse=True)
    # y's error turns with it: at most sqrt 2 of a pair's larger one
    slack = 2 * b1.amax(-1, keepdim=True) + b2.amax(-1, keepdim=True)
    ref.assert_within(back, x.double(), slack.expand_as(back))


def test_in_place_and_views_of_one_buffer():
    """q and k as views of one fused projection, rotated in place; v, between them, is left alone."""
    T, H, W, ids, dims, d = 6, 7, 5, [0, 2, 5], (24, 20, 20), 64
    rows = len(ids) * H * W
    for dtype in (BF16, F32):
        buf = draw((rows, 4 + 2 + 2, d), dtype, 10)
        old = buf.clone()
        q, v, k = buf[:, :4], buf[:, 4:6], buf[:, 6:]
        rf.rf_rotary(q, ids, T, H, W, dims, k=k, out=q, k_out=k)
        for x, y in ((old[:, :4], q), (old[:, 6:], k)):
            want, bound = ref.rotary(x, ids, H, W, dims)
            ref.assert_within(y, want, bound)
        assert torch.equal(v, old[:, 4:6])
        # all frames listed: compact and full are one layout, also in place
        x = draw((2 * 3, 2, d), dtype, 11)
        y = x.clone()
        rf.rf_rotary(y, [0, 1], 2, 1, 3, dims, out=y, in_full=True)
        want, bound = ref.rotary(x, [0, 1], 1, 3, dims)
        ref.assert_within(y, want, bound)


def test_values_that_are_not_numbers_stay_in_their_pair():
    x = draw((6, 2, 32), BF16, 12)
    x[1, 0, 20] = float("inf")      # past R
    x[2, 1, 4] = float("nan")
    y = rf.rf_rotary(x, [0], 1, 2, 3, (4, 4, 2), theta=100.0)
    want, bound = ref.rotary(x, [0], 2, 3, (4, 4, 2), theta=(100.0,) * 3)
    bad = torch.zeros_like(x, dtype=torch.bool)
    bad[2, 1, 4:6] = True
    assert bool(torch.isnan(y[bad]).all()) and float(y[1, 0, 20]) == float("inf")
    bad[1, 0, 20] = True
    ref.assert_within(torch.where(bad, 0, y.double()), torch.where(bad, 0, want), torch.where(bad, 0, bound))


def test_many_heads_few_rows_and_the_reverse():
    for T, H, W, ids, hq, hk, d in ((1, 1, 2, [0], 200, 3, 128), (9, 40, 41, list(range(9)), 1, 1, 8)):
        dims = (4, 2, 2)
        q, k = draw((len(ids) * H * W, hq, d), BF16, 13), draw((len(ids) * H * W, hk, d), BF16, 14)
        y, yk = rf.rf_rotary(q, ids, T, H, W, dims, k=k)
        for a, b in ((q, y), (k, yk)):
            want, bound = ref.rotary(a, ids, H, W, dims)
            ref.assert_within(b, want, bound)


def test_stream_and_graph():
    """On a stream that is not the current one, and captured: every replay equals the eager result."""
    T, H, W, ids, dims = 5, 8, 8, np.array([0, 2, 4], dtype=np.int32), (24, 20, 20)
    x = draw((3 * 64, 2, 64), BF16, 15)
    eager = rf.rf_rotary(x, ids, T, H, W, dims)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y = rf.rf_rotary(x, ids, T, H, W, dims, stream=s)
    s.synchronize()
    assert torch.equal(y, eager)
    out = torch.empty_like(eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rf.rf_rotary(x, ids, T, H, W, dims, out=out)
    for i in range(4):
        x.copy_(draw(x.shape, BF16, 20 + i))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, rf.rf_rotary(x, ids, T, H, W, dims))
