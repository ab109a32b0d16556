"""Norm, rows in 8 bits and their products one after the other, as a block uses them on the listed frames' rows: against
the same chain in 64 bits, on two streams, and captured."""
import pytest
import torch

import block_reference as block
import rows_reference as ref

rf = pytest.importorskip("paper_2606_06309_amd.binding")
pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def draws(seed, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return lambda *shape, scale=1.0: (torch.randn(shape, generator=g, device="cuda", dtype=F32) * scale).to(dtype)


def weights(draw, D):
    """8-bit weights as a program holds them, rounded by the package itself."""
    w = {}
    for name, n, k in (("qkv", 3 * D, D), ("out", D, D), ("up", 4 * D, D), ("down", D, 4 * D)):
        w[name] = rf.rf_frame_quantize(draw(n, k, scale=k ** -0.5))
    return w


def layer(c, full, spaces=None):
    """norm -> 8 bits -> q, k, v -> attention over all frames -> 8 bits -> out, gate and residual -> norm -> 8 bits ->
    up -> 8 bits -> down, all on the listed frames of `full`, which is updated in place."""
    T, H, W, ids, heads, d = c["T"], c["H"], c["W"], c["ids"], c["heads"], c["d"]
    N, D = H * W, heads * d
    kw = dict(frame_ids=ids, T=T, rows_per_frame=N)
    space = lambda name: None if spaces is None else spaces[name]  # noqa: E731
    w = c["w"]
    x8 = rf.rf_frame_group_norm(full, c["groups"], c["nw"], c["nb"], in_full=True, int8=True, workspace=space("norm"), **kw)
    qkv = rf.rf_frame_linear_i8(*x8, *w["qkv"], c["b_qkv"], workspace=space("qkv"), **kw).view(-1, 3, heads, d)
    q, k, v = (torch.zeros((T * N, heads, d), dtype=full.dtype, device="cuda"), c["k"].clone(), c["v"].clone())
    for t, dst in ((0, q), (1, k), (2, v)):
        rf.rf_scatter_frames(qkv[:, t].contiguous(), dst, ids, T, N)
    o = rf.rf_keyframe_attention(q, k, v, ids, T, H, W)
    o8 = rf.rf_frame_quantize(o.view(-1, D), **kw)
    rf.rf_frame_linear_i8(*o8, *w["out"], c["b_out"], gate=c["gate"], residual=full, out=full, out_full=True,
                          workspace=space("out"), **kw)
    # (rows of 8 bits at full positions this time)
    y8 = (torch.full((T * N, D), 3, dtype=torch.int8, device="cuda"), torch.full((T * N,), 2.0, device="cuda"))
    rf.rf_frame_group_norm(full, c["groups"], c["nw"], c["nb"], activation="silu", in_full=True, out_full=True, out=y8[0],
                           out_scale=y8[1], frames_together=len(ids), workspace=space("norm"), **kw)
    u = rf.rf_frame_linear_i8(*y8, *w["up"], c["b_up"], "gelu_tanh", in_full=True, dtype=full.dtype, workspace=space("up"), **kw)
    u8 = rf.rf_frame_quantize(u)
    return rf.rf_frame_linear_i8(*u8, *w["down"], residual=full, out=full, out_full=True, workspace=space("down"), **kw)


def wide(c, full):
    """The same in 64 bits, but for the roundings to 8 bits, which are part of the definitions."""
    T, H, W, ids, heads, d, G = c["T"], c["H"], c["W"], c["ids"], c["heads"], c["d"], c["groups"]
    N, D, M = H * W, heads * d, len(ids)
    pos, sel = block.positions(ids, N, "cuda"), torch.tensor(ids, device="cuda")
    h = full.double()[pos]

    def eight(x):
        q, s = ref.rows8(x)
        return q.cuda(), s.cuda()

    def lin(x8, name, bias=None, act="none", gate=None, residual=None):
        return ref.linear_i8(*x8, *c["w"][name], bias, act, gate, residual)[0]
    n = ref.group_norm(h.view(M, N, D), G, c["nw"][sel], c["nb"][sel])[0].view(-1, D)
    qkv = lin(eight(n), "qkv", c["b_qkv"]).view(-1, 3, heads, d)
    k, v = c["k"].double(), c["v"].double()
    k[pos], v[pos] = qkv[:, 1], qkv[:, 2]
    o = torch.empty((M * N, heads, d), dtype=torch.float64, device="cuda")
    for i in range(heads):
        s = torch.mm(qkv[:, 0, i].contiguous(), k[:, i].t().contiguous()) * d ** -0.5
        o[:, i] = torch.mm(torch.softmax(s, -1), v[:, i])
    h = lin(eight(o.view(-1, D)), "out", c["b_out"], gate=c["gate"][sel].repeat_interleave(N, 0), residual=h)
    n = ref.group_norm(h.view(M, N, D), G, c["nw"][sel], c["nb"][sel], act="silu", together=M)[0].view(-1, D)
    u = lin(eight(n), "up", c["b_up"], "gelu_tanh")
    return lin(eight(u), "down", residual=h)


def setting(seed, dtype, T=5, H=8, W=8, ids=(0, 2, 4), heads=2, d=64, groups=8):
    draw = draws(seed, dtype)
    D, S = heads * d, T * H * W
    return dict(T=T, H=H, W=W, ids=list(ids), heads=heads, d=d, groups=groups, w=weights(draw, D), b_qkv=draw(3 * D),
                b_out=draw(D), b_up=draw(4 * D), gate=draw(T, D), nw=(1 + 0.1 * draw(T, D)).to(dtype), nb=draw(T, D, scale=0.1),
                k=draw(S, heads, d), v=draw(S, heads, d)), draw(S, D)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("size", [dict(), dict(T=7, H=9, W=13, ids=(0, 5), heads=3, d=128, groups=32)])
def test_layer(size, dtype):
    c, full = setting(3, dtype, **size)
    old = full.clone()
    want = wide(c, full)
    layer(c, full)
    pos = block.positions(c["ids"], c["H"] * c["W"], "cuda")
    other = torch.ones(full.shape[0], dtype=torch.bool, device="cuda")
    other[pos] = False
    assert torch.equal(full[other], old[other])
    # Four rounds of 8 bits. A value off by e of its row's step moves to the next whole number with a chance of e, which
    # moves it by a step, 1 / 127 of the row's largest (about 4 deviations: 1 / 32 of one). bf16 rounds eight results,
    # 2^-8 of each: an eighth of a step, so an eighth of the values move by a step, rms 2^-5 / sqrt 8 = 2^-6.5, next to
    # 2^-8 itself; twice that for each of the four products' inputs, and the chain's own gain of at most 2. In fp32
    # 2^-19 of a step, rms 2^-5 * 2^-9.5.
    rel = float(torch.linalg.norm(full[pos].double() - want) / torch.linalg.norm(want))
    assert rel <= {BF16: 8 * 2.0 ** -6.5, F32: 8 * 2.0 ** -14.5}[dtype], rel


def spaces_of(c, dtype):
    M, N, D = len(c["ids"]), c["H"] * c["W"], c["heads"] * c["d"]
    need = {"norm": max(rf.rf_frame_group_norm_workspace(M, N, D, c["groups"], dtype, True, t) for t in (1, M))}
    for name, n, k in (("qkv", 3 * D, D), ("out", D, D), ("up", 4 * D, D), ("down", D, 4 * D)):
        need[name] = rf.rf_frame_linear_i8_workspace(M, N, k, n, dtype)
    return {n: torch.empty(max(16, b), dtype=torch.uint8, device="cuda") for n, b in need.items()}


def test_two_streams_at_once():
    sets = [setting(10 + i, BF16, T=9, H=20, W=30, ids=(0, 4, 8)) for i in range(2)]
    alone = []
    for c, full in sets:
        h = full.clone()
        layer(c, h)
        alone.append(h)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(4):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                h = sets[i][1].clone()
                layer(sets[i][0], h)
                got[i].append(h)
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(h, alone[i]) for h in got[i])


def test_stream_argument():
    """The operators on a stream that is not the current one, their outputs and workspaces allocated for it."""
    draw = draws(20, BF16)
    x, w = draw(3000, 320), rf.rf_frame_quantize(draw(320, 320))

    def run(stream=None):
        n = rf.rf_frame_group_norm(x, 32, stream=stream)
        n8 = rf.rf_frame_group_norm(x, 32, int8=True, stream=stream)
        y = rf.rf_frame_linear_i8(*n8, *w, stream=stream)
        return n, *n8, y, *rf.rf_frame_quantize(x, stream=stream)
    want = run()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for stream in (s, s.cuda_stream):
        got = run(stream)
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_two_graphs_with_workspaces_of_their_own():
    """Captured layers replayed in turn and at once on two streams, eager work between, against the eager result."""
    graphs, outs, want, keep = [], [], [], []
    for i in range(2):
        c, full = setting(30 + i, BF16, T=6, H=16, W=20, ids=(1, 3, 5), groups=16)
        spaces = spaces_of(c, BF16)
        eager = full.clone()
        layer(c, eager, spaces)
        torch.cuda.synchronize()
        h = full.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            layer(c, h, spaces)
        graphs.append(graph)
        outs.append((h, full))
        want.append(eager)
        keep.append((c, spaces))
    streams = [torch.cuda.Stream() for _ in range(2)]
    for turn in range(4):
        for h, full in outs:
            h.copy_(full)
        keep[0][1]["norm"].fill_(turn)     # what a workspace holds before means nothing
        rf.rf_frame_group_norm(outs[0][1], 16)
        torch.cuda.synchronize()
        for i in range(2):
            with torch.cuda.stream(streams[i] if turn % 2 else torch.cuda.current_stream()):
                graphs[i].replay()
        torch.cuda.synchronize()
        for (h, _), eager in zip(outs, want):
            assert torch.equal(h, eager)


def test_norm_and_rounding_agree():
    """A norm into 8 bits is the norm's fp32 rows, rounded: the same but where the norms differ in their last places."""
    x = draws(40, F32)(3 * 700, 256)
    kw = dict(frame_ids=[0, 1, 2], T=3, rows_per_frame=700, activation="silu")
    q, s = rf.rf_frame_group_norm(x, 32, int8=True, **kw)
    q2, s2 = rf.rf_frame_quantize(rf.rf_frame_group_norm(x, 32, **kw))
    assert float(((s - s2).abs() / s2).max()) < 1e-5
    assert int((q.int() - q2.int()).abs().max()) <= 1 and float((q != q2).float().mean()) < 1e-3
