"""A block at a skipped step: the operators one after the other, as they are used, against the same chain in 64 bits."""
import math

import pytest
import torch

import block_reference as ref

rf = pytest.importorskip("paper_2606_06309_amd.binding")
pytestmark = pytest.mark.gpu


def chain(c, wide):
    """The block on tensors c; wide=True in 64 bits from the definitions, else through the package."""
    T, H, W, ids, heads, d, dims = c["T"], c["H"], c["W"], c["ids"], c["heads"], c["d"], c["dims"]
    N, D = H * W, heads * d
    pos = ref.positions(ids, N, c["h"].device)
    sel = torch.tensor(ids, device=c["h"].device)
    if wide:
        f = {n: (t.double() if isinstance(t, torch.Tensor) and t.is_floating_point() else t) for n, t in c.items()}

        def lin(x, w, b=None, act="none", gate=None, res=None):
            return ref.linear(x, f[w], f[b] if b else None, act, gate, res)[0]
        h = f["h"][pos]
        qkv = lin(h, "w_qkv", "b_qkv").view(-1, 3, heads, d)
        q = ref.rotary(qkv[:, 0], ids, H, W, dims)[0]
        k_full, v_full = f["k"].clone(), f["v"].clone()
        k_full[pos], v_full[pos] = ref.rotary(qkv[:, 1], ids, H, W, dims)[0], qkv[:, 2]
        o = torch.empty_like(q)
        for i in range(heads):
            s = torch.mm(q[:, i], k_full[:, i].t().contiguous()) / math.sqrt(d)
            o[:, i] = torch.mm(torch.softmax(s, -1), v_full[:, i])
        h = lin(o.reshape(-1, D), "w_o", "b_o", gate=f["gate"][sel].repeat_interleave(N, 0), res=h)
        qc = lin(h, "w_cq").view(1, -1, heads, d)
        kv = lin(f["prompt"], "w_ckv").view(1, -1, 2, heads, d)
        x = ref.cross(qc, kv[:, :, 0], kv[:, :, 1], [c["prompt_len"]])[0]
        h = lin(x.reshape(-1, D), "w_co", res=h)
        u = lin(h, "w_up", "b_up", "gelu_tanh")
        return lin(u, "w_down", res=h)
    ids_kw = dict(frame_ids=ids, T=T, rows_per_frame=N)
    full = c["h"].clone()
    qkv = rf.rf_frame_linear(full, c["w_qkv"], c["b_qkv"], in_full=True, **ids_kw).view(-1, 3, heads, d)
    q, k, v = torch.empty_like(c["k"]), c["k"].clone(), c["v"].clone()
    rf.rf_rotary(qkv[:, 0], ids, T, H, W, dims, k=qkv[:, 1], out=q, k_out=k, out_full=True)
    rf.rf_scatter_frames(qkv[:, 2].contiguous(), v, ids, T, N)
    o = rf.rf_keyframe_attention_ws(q, k, v, ids, T, H, W)
    # the gated residual, in place at the keyframes' rows of the full hidden states
    rf.rf_frame_linear(o.view(-1, D), c["w_o"], c["b_o"], gate=c["gate"], residual=full, out=full, out_full=True, **ids_kw)
    qc = rf.rf_frame_linear(full, c["w_cq"], in_full=True, **ids_kw).view(1, -1, heads, d)
    kv = rf.rf_frame_linear(c["prompt"], c["w_ckv"]).view(1, -1, 2, heads, d)
    lengths = torch.tensor([c["prompt_len"]], dtype=torch.int32, device=full.device)
    x = rf.rf_cross_attention(qc, kv[:, :, 0], kv[:, :, 1], lengths)
    rf.rf_frame_linear(x.view(-1, D), c["w_co"], residual=full, out=full, out_full=True, **ids_kw)
    u = rf.rf_frame_linear(full, c["w_up"], c["b_up"], "gelu_tanh", in_full=True, **ids_kw)
    rf.rf_frame_linear(u, c["w_down"], residual=full, out=full, out_full=True, **ids_kw)
    other = torch.ones(T * N, dtype=torch.bool, device=full.device)
    other[pos] = False
    assert torch.equal(full[other], c["h"][other])
    return full[pos]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H,W,ids,heads,d,dims", [(5, 8, 8, [0, 2, 4], 2, 64, (24, 20, 20)),
                                                    (7, 9, 13, [0, 5], 3, 128, (44, 42, 42))])
def test_block(T, H, W, ids, heads, d, dims, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(77)

    def draw(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)
    S, D, L = T * H * W, heads * d, 77
    s = D ** -0.5
    c = dict(T=T, H=H, W=W, ids=ids, heads=heads, d=d, dims=dims, prompt_len=50, h=draw(S, D), k=draw(S, heads, d),
             v=draw(S, heads, d), prompt=draw(L, D), gate=draw(T, D), w_qkv=draw(3 * D, D, scale=s), b_qkv=draw(3 * D),
             w_o=draw(D, D, scale=s), b_o=draw(D), w_cq=draw(D, D, scale=s), w_ckv=draw(2 * D, D, scale=s),
             w_co=draw(D, D, scale=s), w_up=draw(4 * D, D, scale=s), b_up=draw(4 * D), w_down=draw(D, 4 * D, scale=s / 2))
    got, want = chain(c, False).double(), chain(c, True)
    # eight operators, each rounding its output once (bf16 2^-8, fp32 2^-24 and its sums) on values of order one:
    # relative to the whole, 8 half steps and the chain's own gain of at most 2
    half = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -20}[dtype]
    rel = float(torch.linalg.norm(got - want) / torch.linalg.norm(want))
    assert rel <= 16 * half, rel


def test_two_streams_at_once():
    """Calls on two streams, each with a workspace of its own, give what they give one after the other."""
    g = torch.Generator(device="cuda")
    g.manual_seed(5)

    def draw(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)
    sets = []
    for i in range(2):
        q, k, v = draw(2, 3, 8, 128), draw(2, 9000 + i, 2, 128), draw(2, 9000 + i, 2, 128)
        x, w = draw(200, 4096), draw(256, 4096)
        sets.append((q, k, v, x, w))

    def both(s, stream=None):
        q, k, v, x, w = s
        return (rf.rf_cross_attention(q, k, v, stream=stream), rf.rf_frame_linear(x, w, stream=stream))
    alone = [both(s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(5):
        for i in range(2):
            got[i].append(both(sets[i], streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for pair in got[i]:
            for a, b in zip(pair, alone[i]):
                assert torch.equal(a, b)


def test_two_graphs_with_workspaces_of_their_own():
    """Two captured graphs replayed in turn and on two streams at once."""
    g = torch.Generator(device="cuda")
    g.manual_seed(6)

    def draw(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)
    graphs, outs, want, alive = [], [], [], []
    for i in range(2):
        q, k, v = draw(1, 2, 4, 64), draw(1, 12000, 4, 64), draw(1, 12000, 4, 64)
        x, w = draw(100, 6000), draw(128, 6000)
        ws = [torch.empty(max(16, n), dtype=torch.uint8, device="cuda")
              for n in (rf.rf_cross_attention_workspace(1, 2, 12000, 4, 4, 64, torch.bfloat16),
                        rf.rf_frame_linear_workspace(1, 100, 6000, 128, torch.bfloat16))]
        out = (torch.empty_like(q), torch.empty((100, 128), dtype=torch.bfloat16, device="cuda"))
        alive.append((q, k, v, x, w, ws))      # a graph holds addresses, not tensors

        def call(out):
            rf.rf_cross_attention(q, k, v, out=out[0], workspace=ws[0])
            rf.rf_frame_linear(x, w, out=out[1], workspace=ws[1])
        eager = tuple(torch.empty_like(o) for o in out)
        call(eager)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(out)
        graphs.append(graph)
        outs.append(out)
        want.append(eager)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for turn in range(4):
        for out in outs:
            for o in out:
                o.fill_(turn)
        torch.cuda.synchronize()
        for i in range(2):
            with torch.cuda.stream(streams[i] if turn % 2 else torch.cuda.current_stream()):
                graphs[i].replay()
        torch.cuda.synchronize()
        for out, eager in zip(outs, want):
            assert all(torch.equal(a, b) for a, b in zip(out, eager))
