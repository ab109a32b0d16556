"""Matrix products whose tiles hold rows of listed frames that lie more than 2 GB apart in x (offsets past 31 bits), and
more than 4 GB, against their definition in 64 bits."""
import pytest
import torch

import block_reference as ref

rf = pytest.importorskip("paper_2606_06309_amd.binding")
pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
T = 256


def draw(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda", dtype=F32) * scale).to(dtype)


def rows_of_frames(ids, N, K, dtype):
    """x at full positions: random rows of the listed frames, and 3 in all others, so that a wrong row shows."""
    x = torch.full((T * N, K), 3.0, dtype=dtype, device="cuda")
    for i, f in enumerate(ids):
        x[f * N:(f + 1) * N] = draw((N, K), dtype, 100 + i)
    return x


# N: a frame that no tile divides; one of which three meet in a tile (neither neighbour 2 GB away). Rows of 56,800 bytes:
# the last step of the reduction is short. ids: 2.4 GB apart, 4.3 GB, both in one call.
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,ids", [(300, [0, 140]), (300, [0, 255]), (300, [1, 2, 143, 255]), (200, [0, 127, 255]),
                                   (77, [0, 1, 2, 253, 254, 255])])
def test_far_frames(N, ids, dtype):
    row = 56800 if N > 100 else 160080   # bytes
    K, n = row // (4 if dtype == F32 else 2), 136
    assert max((b - a - 1) * N * row for a, b in zip(ids, ids[1:] if N > 255 else ids[2:])) > 2 ** 31
    x, w = rows_of_frames(ids, N, K, dtype), draw((n, K), dtype, 2, K ** -0.5)
    b, gate, full = draw((n,), dtype, 3), draw((T, n), dtype, 4), draw((T * N, n), dtype, 5)
    pos = ref.positions(ids, N, "cuda")
    gates = gate[torch.tensor(ids, device="cuda")].repeat_interleave(N, 0)
    kw = dict(frame_ids=ids, T=T, rows_per_frame=N, in_full=True)
    # the whole epilogue, rows to their positions; the reduction is split where that pays
    want, bound = ref.linear(x[pos], w, b, "silu", gates, full[pos])
    out = full.clone()
    rf.rf_frame_linear(x, w, b, "silu", gate, out, out=out, out_full=True, **kw)
    ref.assert_within(out[pos], want, bound, f"{N} {ids}")
    other = torch.ones(T * N, dtype=torch.bool, device="cuda")
    other[pos] = False
    assert torch.equal(out[other], full[other])
    # without a workspace, so without a split
    y = torch.empty((len(ids) * N, n), dtype=dtype, device="cuda")
    arr, p = rf._ids(ids)
    rf._check(rf.lib.rf_frame_linear(x.data_ptr(), w.data_ptr(), None, None, None, y.data_ptr(), p, len(ids), T, N, K, n, 0,
                                     rf.RF_ROWS_IN_FULL, rf._dtype_code(dtype), None, 0, rf._stream(None)))
    ref.assert_within(y, *ref.linear(x[pos], w), f"{N} {ids} whole")
    # the same rows side by side: no tile is wide, and the products are those of other kernels
    ref.assert_within(rf.rf_frame_linear(x[pos], w, b, "silu", gates[:1], None, frame_ids=[0], T=1,
                                         rows_per_frame=len(ids) * N),
                      *ref.linear(x[pos], w, b, "silu", gates[:1]), f"{N} {ids} compact")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,ids,row", [(300, [0, 140], 56800), (300, [0, 255], 56816), (200, [0, 127, 255], 56832),
                                       (77, [0, 1, 2, 253, 254, 255], 160080), (1, [0, 255], (7 << 20) - 16)])
def test_far_frames_exactly(N, ids, row, dtype):
    """Whole numbers from -2 to 2: every sum is below 4 K < 2^24, so exact in fp32 in any order, and the result is that
    sum, rounded once."""
    K, n = row // (4 if dtype == F32 else 2), 72
    assert 4 * K < 2 ** 24
    x = torch.full((T * N, K), 3.0, dtype=dtype, device="cuda")
    for i, f in enumerate(ids):
        x[f * N:(f + 1) * N] = draw((N, K), F32, 120 + i).round().clamp(-2, 2).to(dtype)
    w = draw((n, K), F32, 8).round().clamp(-2, 2).to(dtype)
    pos = ref.positions(ids, N, "cuda")
    want = torch.mm(x[pos].double(), w.double().t().contiguous()).to(dtype)
    got = rf.rf_frame_linear(x, w, frame_ids=ids, T=T, rows_per_frame=N, in_full=True)
    assert torch.equal(got, want), (N, ids, int((got != want).sum()))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_far_rows_and_features(dtype):
    """Several tiles of rows and features, rows of whole steps, from one frame's rows into those of one 2.1 GB on."""
    N, ids, n = 1560, [0, 1, 30, 31], 520
    K = 24576 // (4 if dtype == F32 else 2) * 2
    assert (28 * N + 127) * K * (4 if dtype == F32 else 2) > 2 ** 31   # a tile of 128 rows, 28 frames between
    x = torch.full((32 * N, K), 3.0, dtype=dtype, device="cuda")
    for i, f in enumerate(ids):
        x[f * N:(f + 1) * N] = draw((N, K), dtype, 110 + i)
    w, r = draw((n, K), dtype, 6, K ** -0.5), draw((len(ids) * N, n), dtype, 7)
    pos = ref.positions(ids, N, "cuda")
    want, bound = ref.linear(x[pos], w, residual=r)
    y = rf.rf_frame_linear(x, w, residual=r, frame_ids=ids, T=32, rows_per_frame=N, in_full=True)
    ref.assert_within(y, want, bound)
