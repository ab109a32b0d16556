"""Attention to an encoder's states against its definition in 64 bits."""
import pytest
import torch

import block_reference as ref

rf = pytest.importorskip("paper_2606_06309_amd.binding")
pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def draw(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda", dtype=F32) * scale).to(dtype)


def make(B, Lq, Lk, heads, kvh, d, dtype, seed=0):
    return (draw((B, Lq, heads, d), dtype, seed), draw((B, Lk, kvh, d), dtype, seed + 1),
            draw((B, Lk, kvh, d), dtype, seed + 2))


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# B, Lq, Lk, heads, kv heads
SIZES = [
    (1, 1, 1, 1, 1), (1, 1, 2, 2, 1), (1, 31, 31, 1, 1), (1, 32, 32, 2, 2), (1, 33, 63, 3, 1), (2, 64, 64, 2, 2),
    (1, 65, 65, 1, 1), (3, 127, 77, 2, 1), (1, 129, 127, 4, 2), (2, 255, 128, 1, 1), (1, 257, 129, 2, 2),
    (1, 300, 512, 5, 5), (5, 17, 200, 6, 3), (1, 1000, 33, 3, 3), (2, 520, 191, 8, 1),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", SIZES)
def test_sizes(size, d, dtype):
    q, k, v = make(*size, d, dtype)
    out = rf.rf_cross_attention(q, k, v)
    ref.assert_within(out, *ref.cross(q, k, v), f"{size} {d}")


# few rows, a long key axis: the key axis is split over workgroups
LONG = [(1, 1, 4097, 2, 2), (2, 1, 20280, 4, 1), (1, 5, 3000, 16, 2), (1, 40, 9001, 1, 1), (3, 2, 1500, 3, 3),
        (1, 64, 32768, 2, 1), (1, 1, 70001, 1, 1)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", LONG)
def test_long_key_axis(size, d, dtype):
    q, k, v = make(*size, d, dtype, seed=3)
    want, bound = ref.cross(q, k, v)
    ref.assert_within(rf.rf_cross_attention(q, k, v), want, bound, f"{size} {d}")
    B, Lk = k.shape[:2]
    lengths = i32([Lk - 1 - 700 * b for b in range(B)])
    mask = draw((B, Lk), F32, 9) > -0.5
    mask[:, 100:900] = False
    ref.assert_within(rf.rf_cross_attention(q, k, v, lengths, mask), *ref.cross(q, k, v, lengths, mask), f"{size} {d}")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Lq", [1, 40, 700])
def test_lengths(Lq, d, dtype):
    """Every length around the tiles' edges, none and too large ones among them; keys past the length are poisoned."""
    lens = [0, 1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300, 500, -3, 10 ** 6]
    Lk = 300
    q, k, v = make(len(lens), Lq, Lk, 2, 1, d, dtype, seed=5)
    want, bound = ref.cross(q, k, v, lens)
    for b, n in enumerate(lens):
        n = max(0, min(n, Lk))
        k[b, n:] = float("nan")
        v[b, n:] = float("inf")
    out = rf.rf_cross_attention(q, k, v, i32(lens))
    ref.assert_within(out, want, bound)
    assert not bool(out[0].any()) and not bool(out[13].any())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Lq", [1, 90, 600])
def test_masks(Lq, d, dtype):
    """Holes, whole tiles of them, single keys at either end, nothing at all; with lengths too. Masked keys and
    values hold infinities and NaN. A mask's bytes are any nonzero value."""
    B, Lk = 7, 333
    q, k, v = make(B, Lq, Lk, 3, 3, d, dtype, seed=6)
    mask = torch.zeros((B, Lk), dtype=torch.uint8, device="cuda")
    mask[0] = 1
    mask[1] = (draw((Lk,), F32, 7) > 0).to(torch.uint8) * 255
    mask[2, Lk - 1] = 2
    mask[3, 0] = 128
    mask[4, 128:256] = 1
    mask[6, 64:] = 1
    lengths = [Lk, 200, Lk, 5, 192, Lk, 64]
    for lens in (None, lengths):
        kk, vv = k.clone(), v.clone()
        ok = mask != 0
        if lens is not None:
            ok &= torch.arange(Lk, device="cuda")[None, :] < i32(lens)[:, None]
        want, bound = ref.cross(q, k, v, lens, mask)
        kk[~ok] = float("-inf")
        vv[~ok] = float("nan")
        out = rf.rf_cross_attention(q, kk, vv, None if lens is None else i32(lens), mask)
        ref.assert_within(out, want, bound)
        assert not bool(out[5].any())
        if lens is not None:
            assert not bool(out[6].any())
    assert torch.equal(rf.rf_cross_attention(q, k, v, None, mask != 0), rf.rf_cross_attention(q, k, v, None, mask))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq", [3, 200])
def test_strides(Lq, dtype):
    """Views of fused projections, [B][heads][L][d] order, a prompt shared by the batch, slices with gaps."""
    B, Lk, heads, d = 2, 150, 4, 64
    qkv = draw((B, Lq, 3, heads, d), dtype, 8)
    kv = draw((B, Lk, 2, heads, d), dtype, 9)
    q, k, v = qkv[:, :, 1], kv[:, :, 0], kv[:, :, 1]
    want, bound = ref.cross(q, k, v)
    ref.assert_within(rf.rf_cross_attention(q, k, v), want, bound)
    t = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in (q, k, v)]
    wide = torch.full((B, heads, Lq, 2 * d), 7.0, dtype=dtype, device="cuda")
    out = wide[..., d:].transpose(1, 2)
    assert rf.rf_cross_attention(*t, out=out) is out
    ref.assert_within(out, want, bound)
    assert bool((wide[..., :d] == 7.0).all())
    shared = [x[:1].expand(B, -1, -1, -1) for x in (k, v)]
    ref.assert_within(rf.rf_cross_attention(q, *shared), *ref.cross(q, *shared))
    gaps = [x[:, ::3] for x in (k, v)]
    ref.assert_within(rf.rf_cross_attention(q, *gaps), *ref.cross(q, *gaps))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq,Lk", [(1, 5000), (50, 640), (400, 640)])
def test_scores_of_any_size(Lq, Lk, dtype):
    """Queries and keys whose scores grow along the keys, fall along them, or lie far from zero: the softmax's
    reference has to move. One row's largest score is the last key's."""
    d, heads = 64, 2
    q, k, v = make(1, Lq, Lk, heads, heads, d, dtype, seed=10)
    ramp = torch.linspace(0.01, 30.0, Lk, device="cuda")[None, :, None, None]
    for kk in ((k.float() * ramp).to(dtype), (k.float() * ramp.flip(1)).to(dtype)):
        ref.assert_within(rf.rf_cross_attention(q, kk, v), *ref.cross(q, kk, v))
    # one common direction: all scores near +-2000, whatever the key
    for sign in (1.0, -1.0):
        q2, k2 = q.clone(), k.clone()
        q2[..., 0], k2[..., 0] = 128.0, sign * 125.0
        ref.assert_within(rf.rf_cross_attention(q2, k2, v), *ref.cross(q2, k2, v))
    k3 = k.clone()
    k3[:, -1] = q[:, 0] * 4
    ref.assert_within(rf.rf_cross_attention(q, k3, v), *ref.cross(q, k3, v))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq,Lk", [(1, 3000), (70, 200), (300, 200)])
def test_scores_at_the_ends_of_the_range(Lq, Lk, dtype):
    """Scores as large as the type's: equal ones share the row evenly; keys of -inf scores count as nothing beside
    ordinary ones, first or last; far lower ones too."""
    d = 64
    big = 1.0e18
    q = torch.zeros((1, Lq, 1, d), dtype=dtype, device="cuda")
    k = torch.zeros((1, Lk, 1, d), dtype=dtype, device="cuda")
    v = draw((1, Lk, 1, d), dtype, 12)
    q[..., 0] = big
    for value in (big, -big):
        k[..., 0] = value          # every score is +-1e36 / 8
        want = v.double().mean(1, keepdim=True).expand(1, Lq, 1, d)
        spread = v.double().abs().mean(1, keepdim=True) + want.abs()
        half = ref.HALF[dtype]
        ref.assert_within(rf.rf_cross_attention(q, k, v), want, spread * (half + (Lk + d) * ref.U) + half * want.abs())
    for first, last in ((0, Lk - 40), (40, Lk)):
        k[..., 0] = -float("inf")
        k[:, first:last, :, 0] = 0
        k[:, first:last, :, 1] = draw((1, last - first, 1), dtype, 13)
        q[..., 1] = 2.0
        out = rf.rf_cross_attention(q, k, v)
        kk, vv, qq = k[:, first:last].clone(), v[:, first:last], q.clone()
        ref.assert_within(out, *ref.cross(qq, kk, vv))
        k[..., 0] = torch.where(torch.isinf(k[..., 0]), torch.full_like(k[..., 0], -1.0e15), k[..., 0])
        ref.assert_within(rf.rf_cross_attention(q, k, v), *ref.cross(qq, kk, vv))


def test_not_a_number_spoils_only_its_rows():
    q, k, v = make(2, 300, 100, 2, 2, 64, BF16, seed=14)
    want, bound = ref.cross(q, k, v)
    q[0, 5, 1] = float("nan")
    out = rf.rf_cross_attention(q, k, v)
    assert bool(torch.isnan(out[0, 5, 1]).all())
    ok = torch.ones(q.shape, dtype=torch.bool, device="cuda")
    ok[0, 5, 1] = False
    ref.assert_within(torch.where(ok, out.double(), want), want, bound)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_workspace_or_none(dtype):
    """With and without a split: both right; a given workspace gives what an allocated one gives, bit for bit, and is
    not written past its size."""
    q, k, v = make(1, 2, 20000, 4, 2, 128, dtype, seed=15)
    need = rf.rf_cross_attention_workspace(1, 2, 20000, 4, 2, 128, dtype)
    assert need > 0
    want, bound = ref.cross(q, k, v)
    a = rf.rf_cross_attention(q, k, v)
    ws = torch.full((need + 4096,), 77, dtype=torch.uint8, device="cuda")
    b = rf.rf_cross_attention(q, k, v, workspace=ws[:need])
    assert torch.equal(a, b) and bool((ws[need:] == 77).all())
    ref.assert_within(a, want, bound)
    import ctypes
    out = torch.empty_like(q)
    rf._check(rf.lib.rf_cross_attention(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), None, None, 1, 2,
                                        20000, 4, 2, 128, None, rf._dtype_code(dtype), None, 0, rf._stream(None)))
    ref.assert_within(out, want, bound)


@pytest.mark.parametrize("size", [(3, 900, 256, 2, 2), (2, 1, 30000, 4, 1), (1, 40, 5000, 3, 3)])
def test_results_repeat(size):
    """The same call gives the same bits: nothing is added in an order of its own."""
    q, k, v = make(*size, 128, BF16, seed=16)
    first = rf.rf_cross_attention(q, k, v)
    for _ in range(3):
        assert torch.equal(first, rf.rf_cross_attention(q, k, v))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Lq,Lk", [(1, 9000), (500, 150)])
def test_stream_and_graph(Lq, Lk, dtype):
    q, k, v = make(2, Lq, Lk, 3, 3, 64, dtype, seed=17)
    lengths = i32([Lk, Lk // 2])
    eager = rf.rf_cross_attention(q, k, v, lengths)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y = rf.rf_cross_attention(q, k, v, lengths, stream=s)
    s.synchronize()
    assert torch.equal(y, eager)
    out = torch.empty_like(q)
    ws = torch.empty(max(16, rf.rf_cross_attention_workspace(2, Lq, Lk, 3, 3, 64, dtype)), dtype=torch.uint8,
                     device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rf.rf_cross_attention(q, k, v, lengths, out=out, workspace=ws)
    for i in range(4):
        q.copy_(draw(q.shape, dtype, 30 + i))
        lengths.copy_(i32([Lk - 7 * i, i]))      # the kernel reads the lengths: a replay follows them
        out.fill_(3.0)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, rf.rf_cross_attention(q, k, v, lengths))


def test_offsets_past_32_bits():
    """A batch whose last sequence lies past 2^32 bytes of q and of k; token strides near the largest."""
    B, Lq, Lk, d = 3, 4, 144, 64
    q = torch.empty((B, 1 << 30), dtype=BF16, device="cuda")[:, :Lq * d].view(B, Lq, 1, d)
    kv = torch.empty((2, 1 << 30), dtype=BF16, device="cuda")
    q.copy_(draw(q.shape, BF16, 18))
    step = (1 << 30) // Lk // 8 * 8
    kv = kv.as_strided((2, Lk, 1, d), (1 << 30, step, d, 1))
    assert step * 2 >= 1 << 23 and step * 2 < 1 << 24
    kv.copy_(draw(kv.shape, BF16, 19))
    k, v = kv[:1].expand(B, -1, -1, -1), kv[1:].expand(B, -1, -1, -1)
    ref.assert_within(rf.rf_cross_attention(q, k, v), *ref.cross(q, k, v))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("masked", [False, True])
def test_runs_of_row_tiles(masked, d, dtype):
    """More tiles of rows than workgroups stay on the device, so each walks several, of sequences of unlike length (one
    without any key) and of rows that end inside a tile; the results' rows stand apart and nothing between them is
    written."""
    B, Lq, Lk, heads = 3, 5000, 130, 7
    q, k, v = make(B, Lq, Lk, heads, heads, d, dtype, seed=30)
    lengths = [Lk, 0, 65]
    mask = (draw((B, Lk), F32, 33) > -0.5) if masked else None
    wide = torch.full((B, Lq, heads, d + 8), 7.0, dtype=dtype, device="cuda")
    out = wide[..., :d]
    rf.rf_cross_attention(q, k, v, i32(lengths), mask, out=out)
    ref.assert_within(out, *ref.cross(q, k, v, i32(lengths), mask))
    assert bool((wide[..., d:] == 7.0).all())
    assert torch.equal(rf.rf_cross_attention(q, k, v, i32(lengths), mask), out)
