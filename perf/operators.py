"""A DiT block's operators around the keyframe attention, at the sizes that they are used at.

  rotary   rotary positions over time, height and width of the queries and keys of the listed frames
  cross    attention to an encoder's states (a prompt's tokens; a clip's tokens for one word of a caption)
  linear   matrix product with bias, activation, gate and residual in its epilogue, on the listed frames' rows

`run` computes them from elementary torch operations in 32 bits, rounded once at the end, or, where `own` is
true, calls the package. `exact` holds their definitions in 64 bits.

Sizes: T frames of H x W tokens of which M, spread evenly, are computed at a skipped step; `heads` heads of
`dim`; `dims` of it turn with the frame, the row and the column. The rows that come in are those of the M frames
only; where `full` is true the rows that go out go to their positions among all T frames' rows, of which the others
stay as they are.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # the smallest workload of the tests, fp32 from end to end: latency
        dict(name="rotary-tiny-f32", op="rotary", dtype="f32", T=5, H=8, W=8, M=3, heads=2, kv_heads=2, dim=64,
             dims="24 20 20", halves=False, full=True, fused=False),
        # a skipped step of a 480p video: the keyframes' rows, as views of one fused projection, to their
        # positions in the buffers that the attention reads
        dict(name="rotary-480p", op="rotary", dtype="bf16", T=21, H=30, W=52, M=6, heads=12, kv_heads=12, dim=128,
             dims="44 42 42", halves=False, full=True, fused=True),
        # a warm-up step of that video: every frame
        dict(name="rotary-480p-all", op="rotary", dtype="bf16", T=21, H=30, W=52, M=21, heads=12, kv_heads=12,
             dim=128, dims="44 42 42", halves=False, full=False, fused=False),
        # one word of a caption reads two clips of 13 frames of 30 x 52 tokens: few rows, a long key axis
        dict(name="cross-token", op="cross", dtype="bf16", B=2, Lq=1, Lk=20280, heads=16, kv_heads=4, dim=128,
             lengths="full", mask=False, fused=False),
        # the tiny workload's three keyframes and a prompt of 77 tokens, fp32
        dict(name="cross-tiny-f32", op="cross", dtype="f32", B=1, Lq=192, Lk=77, heads=2, kv_heads=2, dim=64,
             lengths="full", mask=False, fused=False),
        # a short clip at a ragged size, two images' and prompts' states whose padding is masked, and a third
        # sequence that has no key at all
        dict(name="cross-clip-masked", op="cross", dtype="bf16", B=3, Lq=1581, Lk=334, heads=5, kv_heads=5, dim=64,
             lengths="none", mask=True, fused=False),
        # the 480p video's keyframes with and without their prompt (guidance), padded to 512; keys and values are
        # views of one fused projection
        dict(name="cross-480p", op="cross", dtype="bf16", B=2, Lq=9360, Lk=512, heads=12, kv_heads=12, dim=128,
             lengths="ragged", mask=False, fused=True),
        # six keyframes of the 720p workload over 512 prompt tokens
        dict(name="cross-720p", op="cross", dtype="bf16", B=1, Lq=21600, Lk=512, heads=40, kv_heads=40, dim=128,
             lengths="full", mask=False, fused=False),
        # six frames' own timesteps through the first layer of an embedding: few rows, the weight bounds it
        dict(name="linear-embed", op="linear", dtype="bf16", T=6, N=1, M=6, K=1536, out=9216, act="silu",
             gate="none", residual=False, full=False),
        # the small workload's keyframes through a square layer in fp32
        dict(name="linear-small-f32", op="linear", dtype="f32", T=13, N=1560, M=5, K=1536, out=1536, act="gelu_tanh",
             gate="none", residual=False, full=False),
        # the attention's output projection at a skipped step of the 480p video: the frames' own gates, the
        # residual, rows to their positions
        dict(name="linear-out-480p", op="linear", dtype="bf16", T=21, N=1560, M=6, K=1536, out=1536, act="none",
             gate="frame", residual=True, full=True),
        # the second product of the feed-forward of the 720p workload's six keyframes (40 heads of 128, four
        # times that inside)
        dict(name="linear-down-720p", op="linear", dtype="bf16", T=6, N=3600, M=6, K=20480, out=5120, act="none",
             gate="row", residual=True, full=False),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm."""
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    """One more case: clips of 1 to 33 frames of up to 45 x 80 tokens, 1 to 21,600 rows, 1 to 32,760 keys, 8 to
    20,480 features; odd sizes as often as even ones. No case costs more than the largest listed one."""
    while True:
        op = rng.choice(["rotary", "cross", "cross", "linear", "linear"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        if op == "cross":
            dim = rng.choice([64, 128])
            kv_heads = _log(rng, 1, 40)
            heads = kv_heads * rng.choice([1, 1, 1, 2, 4, 8])
            few = rng.random() < 0.3
            case = dict(op=op, dtype=dtype, B=rng.choice([1, 1, 2, 2, 3, 5]),
                        Lq=_log(rng, 1, 64) if few else _log(rng, 64, 21600),
                        Lk=_log(rng, 256, 32760) if few else _log(rng, 1, 1100), heads=heads, kv_heads=kv_heads,
                        dim=dim, lengths=rng.choice(["none", "full", "ragged", "ragged"]), mask=rng.random() < 0.25,
                        fused=rng.random() < 0.4)
            if heads > 64:
                continue
        elif op == "rotary":
            T, H = _log(rng, 1, 33), _log(rng, 4, 45)
            W = max(4, min(80, round(H * rng.uniform(0.6, 1.9))))
            M = rng.choice([1, max(1, T // 6), max(1, T // 3), T])
            dim = rng.choice([64, 80, 128])
            kv_heads = _log(rng, 1, 24)
            halves = rng.random() < 0.3
            if halves:
                dims = rng.choice(["16 24 24", "0 32 32", "16 8 8", "2 30 32"])
            else:
                h = dim // 6 * 2
                dims = rng.choice([f"{dim - 2 * h} {h} {h}", "16 24 24", "0 10 12", "4 0 0"])
            case = dict(op=op, dtype=dtype, T=T, H=H, W=W, M=M, heads=kv_heads * rng.choice([1, 1, 2, 4]),
                        kv_heads=kv_heads, dim=dim, dims=dims, halves=halves, full=rng.random() < 0.6,
                        fused=rng.random() < 0.4)
        else:
            few = rng.random() < 0.3
            T = _log(rng, 1, 33)
            M = rng.choice([1, max(1, T // 6), max(1, T // 3), T])
            N = _log(rng, 1, 8) if few else _log(rng, 9, 3600)
            case = dict(op=op, dtype=dtype, T=T, N=N, M=M, K=8 * _log(rng, 1, 2560), out=8 * _log(rng, 1, 2560),
                        act=rng.choice(["none", "none", "gelu", "gelu_tanh", "silu"]),
                        gate=rng.choice(["none", "row", "frame"]), residual=rng.random() < 0.5,
                        full=rng.random() < 0.5)
        w = work(case)
        if w["flops"] > (2e11 if dtype == "f32" else 2e12) or w["bytes"] > 5e8:
            continue
        if op == "cross" and 4 * case["B"] * case["Lq"] * case["Lk"] * case["heads"] > 2e9:
            continue
        if op != "cross" and case["T"] * case.get("N", case.get("H", 0) * case.get("W", 0)) * max(
                case.get("out", 0), (case.get("heads", 0) + case.get("kv_heads", 0)) * case.get("dim", 0)) > 3e8:
            continue
        return case


def _frames(T, M):
    """M frames spread evenly over T with both ends among them (the first alone for M = 1)."""
    return [0] if M == 1 else [(2 * i * (T - 1) + M - 1) // (2 * (M - 1)) for i in range(M)]


def _dims(case):
    """Dimensions that turn with the frame, the row and the column."""
    return tuple(int(n) for n in case["dims"].split())


def _lengths(case, seed):
    """Valid keys of each sequence on the host: a prompt fills a part of its padded length, and the prompt of
    guidance is a few tokens."""
    B, Lk = case["B"], case["Lk"]
    if case["lengths"] in ("none", "full"):
        return [Lk] * B
    return [max(1, Lk * (37 + (seed + 13 * b) % 41) // 100) if b % 2 == 0 else min(Lk, 1 + (seed + b) % 9)
            for b in range(B)]


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "rotary":
        n = case["M"] * case["H"] * case["W"] * (case["heads"] + case["kv_heads"]) * case["dim"]
        return {"bytes": 2 * n * size, "flops": 3 * n}
    if case["op"] == "cross":
        keys = sum(_lengths(case, 0))
        rows = case["B"] * case["Lq"] * case["heads"] * case["dim"]
        b = 2 * rows * size + 2 * keys * case["kv_heads"] * case["dim"] * size
        b += case["B"] * case["Lk"] if case["mask"] else 0
        return {"bytes": b, "flops": 4 * case["Lq"] * keys * case["heads"] * case["dim"]}
    rows, K, n = case["M"] * case["N"], case["K"], case["out"]
    b = rows * K + K * n + n + rows * n * (2 if case["residual"] else 1)
    b += {"none": 0, "row": n, "frame": case["M"] * n}[case["gate"]]
    return {"bytes": b * size, "flops": 2 * rows * K * n}


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0):
        # (in parts: the draw itself is in 32 bits)
        x = torch.empty(shape, dtype=dt, device="cuda")
        for part in x.view(-1).split(1 << 27):
            part.copy_(torch.randn(part.shape, generator=g, device="cuda", dtype=torch.float32).mul_(scale))
        return x

    st = {"case": case}
    if case["op"] == "cross":
        B, Lq, Lk, heads, kvh, d = (case[n] for n in ("B", "Lq", "Lk", "heads", "kv_heads", "dim"))
        st["q"] = normal(B, Lq, heads, d)
        if case["fused"]:
            kv = normal(B, Lk, 2, kvh, d)
            st["k"], st["v"] = kv[:, :, 0], kv[:, :, 1]
        else:
            st["k"], st["v"] = normal(B, Lk, kvh, d), normal(B, Lk, kvh, d)
        st["lengths"] = st["mask"] = None
        if case["lengths"] != "none":
            st["lengths"] = torch.tensor(_lengths(case, seed), dtype=torch.int32, device="cuda")
        if case["mask"]:
            # holes as often as keys at the end of each half, and a last sequence without any key
            m = torch.rand((B, Lk), generator=g, device="cuda") < 0.8
            m[:, Lk // 3:Lk // 2] = False
            if B > 2:
                m[B - 1] = False
            st["mask"] = m.to(torch.uint8)
        st["out"] = torch.empty((B, Lq, heads, d), dtype=dt, device="cuda")
        if own:
            from paper_2606_06309_amd import binding as rf
            n = rf.rf_cross_attention_workspace(B, Lq, Lk, heads, kvh, d, dt)
            st["ws"] = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
        return st
    T, M = case["T"], case["M"]
    st["ids"] = _frames(T, M)
    if own:
        import numpy as np
        st["ids"] = np.array(st["ids"], dtype=np.int32)
    if case["op"] == "rotary":
        N, heads, kvh, d = case["H"] * case["W"], case["heads"], case["kv_heads"], case["dim"]
        if case["fused"]:
            x = normal(M * N, heads + 2 * kvh, d)
            st["q"], st["k"] = x[:, :heads], x[:, heads:heads + kvh]
        else:
            st["q"], st["k"] = normal(M * N, heads, d), normal(M * N, kvh, d)
        rows = (T if case["full"] else M) * N
        if case["full"]:
            # the layer's buffers of the step before
            st["q_out"], st["k_out"] = normal(rows, heads, d), normal(rows, kvh, d)
        else:
            st["q_out"] = torch.empty((rows, heads, d), dtype=dt, device="cuda")
            st["k_out"] = torch.empty((rows, kvh, d), dtype=dt, device="cuda")
        return st
    N, K, n = case["N"], case["K"], case["out"]
    st["x"] = normal(M * N, K)
    st["w"] = normal(n, K, scale=1.0 / math.sqrt(K))
    st["bias"] = normal(n, scale=0.3)
    st["gate"] = {"none": lambda: None, "row": lambda: normal(n, scale=0.5),
                  "frame": lambda: normal(T, n, scale=0.5)}[case["gate"]]()
    rows = (T if case["full"] else M) * N
    st["residual"] = normal(rows, n) if case["residual"] else None
    st["y"] = normal(rows, n) if case["full"] else torch.empty((rows, n), dtype=dt, device="cuda")
    return st


def run(st):
    case = st["case"]
    if own:
        return _own(case, st)
    return {"rotary": _rotary, "cross": _cross, "linear": _linear}[case["op"]](case, st)


def _own(case, st):
    from paper_2606_06309_amd import binding as rf
    if case["op"] == "rotary":
        rf.rf_rotary(st["q"], st["ids"], case["T"], case["H"], case["W"], _dims(case), k=st["k"], out=st["q_out"],
                     k_out=st["k_out"], out_full=case["full"], halves=case["halves"])
        return st["q_out"], st["k_out"]
    if case["op"] == "cross":
        return rf.rf_cross_attention(st["q"], st["k"], st["v"], kv_lengths=st["lengths"], key_mask=st["mask"],
                                     out=st["out"], workspace=st["ws"])
    return rf.rf_frame_linear(st["x"], st["w"], st["bias"], activation=case["act"], gate=st["gate"],
                              residual=st["residual"], frame_ids=st["ids"], T=case["T"], rows_per_frame=case["N"],
                              out_full=case["full"], out=st["y"])


def _positions(case, device):
    """The position of every row of the listed frames among all frames' rows."""
    N = case["N"] if "N" in case else case["H"] * case["W"]
    ids = torch.tensor([int(f) for f in _frames(case["T"], case["M"])], device=device)
    return (ids[:, None] * N + torch.arange(N, device=device)[None, :]).reshape(-1)


def _place(case, y, dst):
    """y's rows into dst, at their positions among all frames where the case says so."""
    if case["full"]:
        dst.index_copy_(0, _positions(case, y.device), y.to(dst.dtype))
    else:
        dst.copy_(y)
    return dst


def _angles(case, device):
    """Angle of each row of the listed frames and each pair of dimensions, in 64 bits (position 32 x frequency)."""
    W, N = case["W"], case["H"] * case["W"]
    tok = _positions(case, device)
    axes = (tok // N, tok % N // W, tok % W)
    parts = [axes[a].double()[:, None] * 10000.0 ** (-torch.arange(0, n, 2, device=device, dtype=torch.float64) / n)
             for a, n in enumerate(_dims(case)) if n > 0]
    return torch.cat(parts, dim=1)


def _rotary(case, st):
    phi = _angles(case, st["q"].device)
    cos, sin = phi.cos().float()[:, None, :], phi.sin().float()[:, None, :]
    R = sum(_dims(case))
    out = []
    for name in ("q", "k"):
        x = st[name].float()
        y = x.clone()
        if case["halves"]:
            a, b = x[..., :R // 2], x[..., R // 2:R]
            y[..., :R // 2], y[..., R // 2:R] = a * cos - b * sin, a * sin + b * cos
        else:
            a, b = x[..., 0:R:2], x[..., 1:R:2]
            y[..., 0:R:2], y[..., 1:R:2] = a * cos - b * sin, a * sin + b * cos
        out.append(_place(case, y, st[name + "_out"]))
    return tuple(out)


def _valid(case, st):
    """[B][Lk] truth values of the keys that count."""
    ok = torch.ones((case["B"], case["Lk"]), dtype=torch.bool, device=st["q"].device)
    if st["lengths"] is not None:
        ok &= torch.arange(case["Lk"], device=ok.device)[None, :] < st["lengths"][:, None]
    if st["mask"] is not None:
        ok &= st["mask"] != 0
    return ok


def _cross(case, st):
    group = case["heads"] // case["kv_heads"]
    ok = _valid(case, st)
    for b in range(case["B"]):
        q = st["q"][b].float().transpose(0, 1).contiguous()                             # [heads][Lq][d]
        k = st["k"][b].float().permute(1, 2, 0).repeat_interleave(group, 0).contiguous()   # [heads][d][Lk]
        v = st["v"][b].float().transpose(0, 1).repeat_interleave(group, 0).contiguous()
        s = torch.matmul(q, k) * (1.0 / math.sqrt(case["dim"]))
        s = s.masked_fill(~ok[b], -math.inf)
        top = s.amax(-1, keepdim=True)
        p = (s - top.masked_fill(top == -math.inf, 0.0)).exp()
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p, v * ok[b][None, :, None]) / total.masked_fill(total == 0, 1.0)
        st["out"][b].copy_(o.transpose(0, 1))
    return st["out"]


def _activation(name, x):
    if name == "silu":
        return x / (1.0 + (-x).exp())
    if name == "gelu":
        return 0.5 * x * (1.0 + torch.erf(x * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * x * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x * x * x)))
    return x


def _gate_rows(case, gate):
    """The gate of every row of the listed frames ([1][out] where all rows share one)."""
    if case["gate"] == "row":
        return gate[None, :]
    ids = torch.tensor(_frames(case["T"], case["M"]), device=gate.device)
    return gate[ids].repeat_interleave(case["N"], 0)


def _linear(case, st):
    y = _activation(case["act"], torch.matmul(st["x"].float(), st["w"].float().t()) + st["bias"].float())
    if st["gate"] is not None:
        y = y * _gate_rows(case, st["gate"].float())
    if st["residual"] is not None:
        r = st["residual"].float()
        y = y + (r[_positions(case, y.device)] if case["full"] else r)
    return _place(case, y, st["y"])


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rotary":
        return tuple(_exact_rotary(case, st[n].double(), st[n + "_out"]) for n in ("q", "k"))
    if case["op"] == "cross":
        return _exact_cross(case, st)
    return _exact_linear(case, st)


def _exact_rotary(case, x, dst):
    """Each pair as a complex number, turned by its angle, one frame at a time."""
    H, W, dims = case["H"], case["W"], _dims(case)
    dev, P = x.device, sum(dims) // 2
    freq = [10000.0 ** (-2.0 * j / n) for n in dims for j in range(n // 2)]
    axis = [a for a, n in enumerate(dims) for _ in range(n // 2)]
    out = dst.double()
    for m, f in enumerate(_frames(case["T"], case["M"])):
        part = x[m * H * W:(m + 1) * H * W]
        row = torch.arange(H, device=dev, dtype=torch.float64)[:, None].expand(H, W).reshape(-1)
        col = torch.arange(W, device=dev, dtype=torch.float64)[None, :].expand(H, W).reshape(-1)
        at = (torch.full_like(row, float(f)), row, col)
        phi = torch.stack([at[a] * w for a, w in zip(axis, freq)], 1)[:, None, :]
        turn = torch.polar(torch.ones_like(phi), phi)
        y = part.clone()
        if case["halves"]:
            z = torch.complex(part[..., :P].contiguous(), part[..., P:2 * P].contiguous()) * turn
            y[..., :P], y[..., P:2 * P] = z.real, z.imag
        else:
            z = torch.view_as_complex(part[..., :2 * P].reshape(*part.shape[:-1], P, 2).contiguous()) * turn
            y[..., :2 * P] = torch.view_as_real(z).flatten(-2)
        first = (f if case["full"] else m) * H * W
        out[first:first + H * W] = y
    return out


def _exact_cross(case, st):
    """Head by head over the keys that count only."""
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device=st["q"].device)
    group = case["heads"] // case["kv_heads"]
    for b in range(case["B"]):
        keys = torch.arange(case["Lk"], device=out.device)
        if st["lengths"] is not None:
            keys = keys[:int(st["lengths"][b])]
        if st["mask"] is not None:
            keys = keys[st["mask"][b][keys] != 0]
        if keys.numel() == 0:
            continue
        for h in range(case["heads"]):
            k = st["k"][b, :, h // group].double()[keys]
            v = st["v"][b, :, h // group].double()[keys]
            s = torch.mm(st["q"][b, :, h].double(), k.t().contiguous()) / math.sqrt(case["dim"])
            out[b, :, h] = torch.mm(torch.softmax(s, -1), v)
    return out


def _exact_linear(case, st):
    """Frame by frame."""
    N, out = case["N"], st["y"].double()
    w, bias = st["w"].double().t().contiguous(), st["bias"].double()
    for m, f in enumerate(_frames(case["T"], case["M"])):
        z = torch.mm(st["x"][m * N:(m + 1) * N].double(), w) + bias
        if case["act"] == "silu":
            z = z * torch.sigmoid(z)
        elif case["act"] == "gelu":
            z = z * torch.special.ndtr(z)
        elif case["act"] == "gelu_tanh":
            z = z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3))
        if case["gate"] != "none":
            z = z * (st["gate"] if case["gate"] == "row" else st["gate"][f]).double()
        first = (f if case["full"] else m) * N
        if st["residual"] is not None:
            z = z + st["residual"][first:first + N].double()
        out[first:first + N] = z
    return out
