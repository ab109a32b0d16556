"""Group norm of values whose mean is far from 0 beside their deviations, and of values that do not deviate at all."""
import pytest
import torch

import block_reference as block
import rows_reference as ref

rf = pytest.importorskip("paper_2606_06309_amd.binding")
pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32

# frames, rows of a frame, channels, groups, frames together: norms of one launch and of more; one row and many to a
# thread, one line of threads and many, groups of one channel, of a few and of all, rows that end inside a chunk
SIZES = [(1, 1, 16, 4, 1), (1, 70, 64, 8, 1), (1, 192, 128, 8, 1), (1, 700, 32, 1, 1), (3, 527, 320, 32, 1), (6, 40, 160, 5, 6),
         (1, 1000, 48, 48, 1), (1, 2000, 8192, 32, 1), (1, 5000, 320, 32, 1), (1, 20011, 16, 1, 1), (4, 900, 640, 5, 2),
         (64, 300, 512, 32, 1), (90, 700, 640, 32, 90), (2, 3000, 2080, 5, 1), (1, 30011, 48, 3, 1)]
CONSTANTS = [100.1, -1000.1, 4321.987, -99999.7, 0.1, 1e-3 / 3, 10000.3, 2.0 ** 39 / 3]


def norm(x, groups, M, N, together, **kw):
    return rf.rf_frame_group_norm(x, groups, frame_ids=range(M), T=M, rows_per_frame=N, frames_together=together, **kw)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,N,C,G,together", SIZES)
def test_constants_of_all_bits(M, N, C, G, together, dtype):
    """No deviation: the bias and nothing else, whatever the constant, and rows of zeros in 8 bits."""
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    bias = torch.randn(C, generator=g, device="cuda").to(dtype)
    for turn in range(2):
        value = torch.tensor([CONSTANTS[(i * (1 + turn * 2) + turn) % len(CONSTANTS)] for i in range(G)], device="cuda").to(dtype)
        x = value.repeat_interleave(C // G).expand(M * N, C).contiguous()
        assert torch.equal(norm(x, G, M, N, together, bias=bias), bias.expand(M * N, C))
        assert not bool(norm(x, G, M, N, together).any())
        q, s = norm(x, G, M, N, together, int8=True)
        assert not bool(q.any()) and not bool(s.any())


def around_the_mean(x, groups, weight, bias, eps, together):
    """The definition in 64 bits of fp32 x [M][N][C], and a bound that goes by the deviations.

    D is a group's largest deviation, A its largest magnitude, s = sqrt(var + eps). Sums go over differences of at most
    2 D: of eight rows (8 u 2 D), in joins of means (four roundings of u 2 D each, 15 joins of a thread and 8 of threads
    at most) or, where a workgroup has all rows, of at most 42 values one after the other; channels and parts are joined in 64
    bits. A mean is two numbers, the second off by u of itself, which is u A at most in each of the joins: 64 u^2 A. So
    deviations are off by 100 u 2 D + 64 u^2 A, 1 / s by as much over s and by 46 u more, relative."""
    x = x.double()
    M, N, C = x.shape
    mean, var, A = (t.repeat_interleave(C // groups, 1).repeat_interleave(together, 0)[:, None]
                    for t in ref.moments(x, groups, together))
    d, s = x - mean, torch.sqrt(var + eps)
    D = d.abs().reshape(M // together, together * N, groups, C // groups).amax((1, 3))
    D = D.repeat_interleave(C // groups, 1).repeat_interleave(together, 0)[:, None]
    y = d / s * weight.double()
    off = (200 * D + 64 * ref.U * A) / s
    err = ref.U * (off * weight.double().abs() + y.abs() * (off + 46))
    y = y + bias.double()
    # (the two numbers of a mean, times weight / s, and the bias are three terms, rounded as they are added)
    err = err + 2 * ref.U * (y.abs() + bias.double().abs() + 2 * ref.U * A / s * weight.double().abs())
    return y.view(-1, C), err.view(-1, C)


@pytest.mark.parametrize("eps", [1e-5, 1e-12])
@pytest.mark.parametrize("M,N,C,G,together", SIZES)
def test_few_last_places_around_a_mean(M, N, C, G, together, eps):
    """fp32 values a few of their last places from their mean: as far off as such deviations are, not as the mean is."""
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    value = torch.tensor([CONSTANTS[i % len(CONSTANTS)] for i in range(G)], device="cuda").repeat_interleave(C // G)
    steps = torch.randint(-3, 4, (M * N, C), generator=g, device="cuda", dtype=torch.int32)
    x = (value.expand(M * N, C).contiguous().view(torch.int32) + steps).view(F32)
    w, b = torch.randn(C, generator=g, device="cuda"), torch.randn(C, generator=g, device="cuda")
    y, err = around_the_mean(x.view(M, N, C), G, w, b, eps, together)
    block.assert_within(norm(x, G, M, N, together, weight=w, bias=b, eps=eps), y, err)


@pytest.mark.parametrize("mean", [1e4, -3e6])
@pytest.mark.parametrize("M,N,C,G,together", SIZES + [(3, 21000, 512, 512, 1), (100, 400, 1024, 64, 100)])
def test_deviations_around_a_large_mean(M, N, C, G, together, mean):
    """Deviations near 1, frames and rows that drift, the first value far from the others."""
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = torch.randn((M * N, C), generator=g, device="cuda")
    x += torch.linspace(-1, 1, M * N, device="cuda")[:, None]
    x[0, 0] = 30.0
    x += mean
    w, b = torch.randn(C, generator=g, device="cuda"), torch.randn(C, generator=g, device="cuda")
    y, err = around_the_mean(x.view(M, N, C), G, w, b, 1e-5, together)
    block.assert_within(norm(x, G, M, N, together, weight=w, bias=b), y, err)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,N,C,G,together", SIZES)
@pytest.mark.parametrize("int8", [False, True])
def test_a_workspace_of_exactly_its_bytes(M, N, C, G, together, int8, dtype):
    """Whatever it held before; nothing behind it is written."""
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    x = (torch.randn((M * N, C), generator=g, device="cuda") + 100.0).to(dtype)
    need = rf.rf_frame_group_norm_workspace(M, N, C, G, dtype, int8=int8, frames_together=together)
    runs = []
    for fill in (0, 255):       # (the second: NaN in every place)
        space = torch.full((need + 256,), fill, dtype=torch.uint8, device="cuda")
        got = norm(x, G, M, N, together, int8=int8, workspace=space[:need] if need else None)
        runs.append(got if int8 else (got,))
        assert bool((space[need:] == fill).all())
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_a_captured_norm_of_fp32_rows():
    """Replayed on other rows, with eager norms between."""
    M, N, C, G = 3, 2000, 320, 32
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    draws = [torch.randn((M * N, C), generator=g, device="cuda") + 1000.0 * i for i in range(4)]
    want = [norm(x, G, M, N, 1, activation="silu") for x in draws]
    x, out = draws[0].clone(), torch.empty_like(draws[0])
    space = torch.empty(rf.rf_frame_group_norm_workspace(M, N, C, G, F32), dtype=torch.uint8, device="cuda")
    norm(x, G, M, N, 1, activation="silu", out=out, workspace=space)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm(x, G, M, N, 1, activation="silu", out=out, workspace=space)
    for turn in range(3):
        for i in (1, 3, 0, 2):
            x.copy_(draws[i])
            graph.replay()
            again = norm(draws[i], G, M, N, 1, activation="silu")
            torch.cuda.synchronize()
            assert torch.equal(out, want[i]) and torch.equal(again, want[i]), (turn, i)
