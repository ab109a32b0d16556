"""Rotary positions where a launch has more threads than one axis of a grid takes."""
import pytest
import torch

import block_reference as ref

rf = pytest.importorskip("paper_2606_06309_amd.binding")
pytestmark = pytest.mark.gpu


def test_more_than_2_to_32_threads():
    """Every frame of 4 of 8,192 x 8,192 tokens, one head of 128, in place (69 GB): 16 threads to a token. The rows at both
    ends of the first and last frames are checked, and that dimensions behind the turning ones stay."""
    T, H, W, d, dims = 4, 8192, 8192, 128, (40, 42, 40)
    N = H * W
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("less than 80 GB free")
    x = torch.empty((T * N, 1, d), dtype=torch.bfloat16, device="cuda")
    for part in x.split(N // 4):
        part.fill_(1.5)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    spots = []
    for f in (0, T - 1):
        for rows in ((0, 2), (H // 2, 1), (H - 1, 1)):   # whole rows of the grid
            at = f * N + rows[0] * W
            x[at:at + rows[1] * W] = torch.randn((rows[1] * W, 1, d), generator=g, device="cuda").to(x.dtype)
            spots.append((f, rows[0], rows[1], x[at:at + rows[1] * W].clone()))
    assert rf.rf_rotary(x, list(range(T)), T, H, W, dims, out=x) is x
    for f, row, n, old in spots:
        at = f * N + row * W
        want, bound = ref.rotary(old, [f], n, W, dims, origin=(0.0, float(row), 0.0))
        ref.assert_within(x[at:at + n * W], want, bound, f"frame {f} row {row}")
        assert torch.equal(x[at:at + n * W, :, sum(dims):], old[..., sum(dims):])
    # between them too: a token whose neighbours are all 1.5
    for f, y, c in ((1, 4000, 17), (2, 8191, 8191), (3, 2, 5000)):   # (none in the rows above)
        at = f * N + y * W + c
        want, bound = ref.rotary(torch.full((1, 1, d), 1.5, dtype=x.dtype, device="cuda"), [0], 1, 1, dims,
                                 origin=(float(f), float(y), float(c)))
        ref.assert_within(x[at:at + 1], want, bound, f"token {f} {y} {c}")
    del x
    torch.cuda.empty_cache()
