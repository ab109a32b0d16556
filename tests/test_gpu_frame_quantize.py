"""Rows in 8 bits against their definition, bit by bit."""
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


def same(got, want):
    q, s = got
    wq, ws = want
    assert torch.equal(q.cpu(), wq)
    assert torch.equal(s.cpu().view(torch.int32)[~torch.isnan(ws)], ws.view(torch.int32)[~torch.isnan(ws)])
    assert torch.equal(torch.isnan(s.cpu()), torch.isnan(ws))


SIZES = [(1, 16), (3, 32), (5, 48), (1, 64), (33, 80), (31, 128), (257, 256), (7, 512), (100, 528), (64, 1536), (9, 2048),
         (5, 2064), (130, 4096), (3, 8192), (2, 8208), (3, 20480), (2, 32768), (1, 32784), (2, 65536)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,K", SIZES)
def test_sizes(rows, K, dtype):
    x = draw((rows, K), dtype, rows + K)
    x[:, K // 3] *= 9
    same(rf.rf_frame_quantize(x), ref.rows8(x))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("K", [64, 1024, 4096])
def test_ties_and_extremes(K, dtype):
    """Halves go to the even neighbour; the largest finite row, rows about the smallest that counts, zeros, signed zeros."""
    x = torch.zeros((12, K), dtype=F32, device="cuda")
    half = torch.arange(K, device="cuda").float() % 254 - 127 + 0.5
    x[0], x[0, 0] = half, 127.0            # scale 1: every other value a tie
    x[1], x[1, -1] = half / 4, -127.0 / 4
    x[2] = 3.3e38
    x[3, 5] = -3.0e38
    x[4] = 2.0 ** -100
    x[5] = 2.0 ** -101
    x[6, 3] = 2.0 ** -126
    x[7, 1] = 2.0 ** -140
    x[8, 2] = -0.0
    x[9], x[9, 7] = 2.0 ** -108, 2.0 ** -100
    x[10, K - 1] = 1e-20
    x = x.to(dtype)
    same(rf.rf_frame_quantize(x), ref.rows8(x))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("K", [32, 1536, 5120, 40960])
def test_not_finite(K, dtype):
    """A row with an infinity or a NaN (either sign, any payload, first or last) has scale NaN and q 0; others do not see it."""
    x = draw((8, K), dtype, 3)
    x[1, 0], x[2, K - 1], x[4, K // 2], x[6, 1] = float("inf"), float("-inf"), float("nan"), float("inf")
    x[6, 2] = float("nan")
    bits = x.view(torch.int16 if dtype == BF16 else torch.int32)
    bits[7, 3] = -1                        # a NaN of all ones
    q, s = rf.rf_frame_quantize(x)
    same((q, s), ref.rows8(x))
    assert torch.isnan(s).tolist() == [False, True, True, False, True, False, True, True]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("in_full,out_full", [(False, False), (False, True), (True, False), (True, True)])
@pytest.mark.parametrize("N", [1, 7, 130])
def test_frames(N, in_full, out_full, dtype):
    """Listed rows only; a row stride longer than the row; rows of other frames stay."""
    T, ids, K = 6, [0, 2, 5], 272
    pos = block.positions(ids, N, "cuda")
    wide = draw((T * N if in_full else 3 * N, K + 48), dtype, 4)
    x = wide[:, 16:16 + K]
    rows = x[pos] if in_full else x
    if in_full:
        other = torch.ones(T * N, dtype=torch.bool, device="cuda")
        other[pos] = False
        wide[other] = float("nan")
        rows = x[pos]
    n = T * N if out_full else 3 * N
    q, s = torch.full((n, K), 77, dtype=torch.int8, device="cuda"), torch.full((n,), 5.0, device="cuda")
    got = rf.rf_frame_quantize(x, frame_ids=ids, T=T, rows_per_frame=N, in_full=in_full, out_full=out_full, out=q, out_scale=s)
    assert got[0] is q and got[1] is s
    same((q[pos], s[pos]) if out_full else (q, s), ref.rows8(rows.contiguous()))
    if out_full:
        other = torch.ones(T * N, dtype=torch.bool, device="cuda")
        other[pos] = False
        assert bool((q[other] == 77).all()) and bool((s[other] == 5.0).all())


def test_rows_far_apart():
    """Rows 1.5 GB apart."""
    K, stride = 48, (1 << 30) * 3 // 4
    x = torch.empty(3 * stride + K, dtype=BF16, device="cuda").as_strided((4, K), (stride, 1))
    x.copy_(draw((4, K), BF16, 5))
    same(rf.rf_frame_quantize(x), ref.rows8(x.contiguous()))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_rows(dtype):
    """More rows than a launch has workgroups for at once."""
    x = draw((300001, 32), dtype, 6)
    same(rf.rf_frame_quantize(x), ref.rows8(x))
