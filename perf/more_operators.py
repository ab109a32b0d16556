"""Normalisation and 8-bit products of the listed frames' rows, at the sizes that they are used at.

  norm      group norm with an activation, channels last: statistics of a frame's rows, or of all listed frames' together
  linear8   matrix product in 8-bit integers, a scale for each row and each output feature, with bias, activation,
            gate and residual; the rows arrive in 8 bits (`given`) or are rounded to them first
  norm8     group norm whose rows leave in 8 bits, and the 8-bit product that reads them

`run` computes them from elementary torch operations in 32 bits, rounded once at the end, or, where `own` is
true, calls the package. `exact` holds their definitions in 64 bits.

Sizes: T frames of N rows of which M, spread evenly, are computed at a skipped step. The rows that come in are those
of the M frames only; where `full` is true the rows that go out go to their positions among all T frames' rows, of
which the others stay as they are.

A row in 8 bits: scale = max |x| / 127 and q = x * (127 / max |x|) to the nearest whole number, ties to even, each of
the three results in fp32 (rows whose largest magnitude is below 2^-100 are zeros).
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def listed():
    return [
        # the tests' smallest clip, fp32 from end to end: latency
        dict(name="norm-tiny-f32", op="norm", dtype="f32", T=5, N=64, M=3, C=128, groups=32, act="silu", affine="one",
             together=False, full=True),
        # a short clip at a ragged size (17 x 31 tokens) before its projection: ten channels to a group
        dict(name="norm-clip", op="norm", dtype="bf16", T=9, N=527, M=3, C=320, groups=32, act="none", affine="one",
             together=False, full=False),
        # six of 21 frames of 30 x 52, whose timesteps are their own: scale and shift for each frame
        dict(name="norm-480p", op="norm", dtype="bf16", T=21, N=1560, M=6, C=640, groups=32, act="silu",
             affine="frame", together=False, full=True),
        # a level of a decoder of latents, 5 frames of 120 x 208, normalised over time as well
        dict(name="norm-decode-clip", op="norm", dtype="bf16", T=5, N=24960, M=5, C=512, groups=32, act="silu",
             affine="one", together=True, full=False),
        # the last level of a decoder: 4 frames of 480 x 832 pixels
        dict(name="norm-decode-480p", op="norm", dtype="bf16", T=4, N=399360, M=4, C=128, groups=32, act="silu",
             affine="one", together=False, full=False),
        # six frames' own timesteps through the first layer of an embedding: few rows, the weight bounds it
        dict(name="linear8-embed", op="linear8", dtype="bf16", T=6, N=1, M=6, K=1536, out=9216, act="silu",
             gate="none", residual=False, full=False, given=False),
        # a clip's three keyframes at sizes that divide no tile, results in fp32
        dict(name="linear8-ragged-f32", op="linear8", dtype="f32", T=9, N=527, M=3, K=1360, out=1004, act="gelu",
             gate="row", residual=True, full=True, given=False),
        # the attention's output projection at a skipped step of the 480p video: the frames' own gates, the
        # residual, rows to their positions
        dict(name="linear8-out-480p", op="linear8", dtype="bf16", T=21, N=1560, M=6, K=1536, out=1536, act="none",
             gate="frame", residual=True, full=True, given=False),
        # the feed-forward's first product there; its rows have been rounded for another product already
        dict(name="linear8-up-480p", op="linear8", dtype="bf16", T=21, N=1560, M=6, K=1536, out=6144,
             act="gelu_tanh", gate="none", residual=False, full=False, given=True),
        # the second product of the feed-forward of the 720p workload's six keyframes
        dict(name="linear8-down-720p", op="linear8", dtype="bf16", T=6, N=3600, M=6, K=20480, out=5120, act="none",
             gate="row", residual=True, full=False, given=False),
        # the ragged clip's norm and projection, one after the other
        dict(name="norm8-clip", op="norm8", dtype="bf16", T=9, N=527, M=3, C=320, groups=32, out=320, full=False),
        # the same of the 480p video's keyframes at the width of its blocks, rows to their positions
        dict(name="norm8-480p", op="norm8", dtype="bf16", T=21, N=1560, M=6, C=1536, groups=32, out=1536, full=True),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm."""
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _groups(rng, C):
    """A number of groups that divides C: its largest divisors up to 128, and 8, 16 and 32 where they do."""
    return rng.choice([g for g in range(1, min(C, 128) + 1) if C % g == 0][-4:] + [g for g in (8, 16, 32) if C % g == 0])


def draw(rng):
    """One more case: clips of 1 to 33 frames, 1 to 60,000 rows a frame under a norm and 1 to 3,600 under a product, 8
    to 2,560 channels, 16 to 20,480 features; odd sizes as often as even ones. No case costs more than the largest
    listed one."""
    while True:
        op = rng.choice(["norm", "norm", "linear8", "linear8", "norm8"])
        T = _log(rng, 1, 33)
        M = rng.choice([1, max(1, T // 6), max(1, T // 3), T])
        full = rng.random() < 0.5
        if op == "norm":
            C = 8 * _log(rng, 1, 320)
            case = dict(op=op, dtype=rng.choice(["bf16", "bf16", "f32"]), T=T, N=_log(rng, 1, 60000), M=M, C=C,
                        groups=_groups(rng, C), act=rng.choice(["none", "silu", "silu", "gelu", "gelu_tanh"]),
                        affine=rng.choice(["none", "one", "one", "frame"]), together=rng.random() < 0.3, full=full)
        elif op == "linear8":
            few = rng.random() < 0.3
            case = dict(op=op, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), T=T,
                        N=_log(rng, 1, 8) if few else _log(rng, 9, 3600), M=M, K=16 * _log(rng, 1, 1280),
                        out=8 * _log(rng, 1, 2560), act=rng.choice(["none", "none", "gelu", "gelu_tanh", "silu"]),
                        gate=rng.choice(["none", "row", "frame"]), residual=rng.random() < 0.5, full=full,
                        given=rng.random() < 0.4)
        else:
            C = 16 * _log(rng, 1, 160)
            case = dict(op=op, dtype="bf16", T=T, N=_log(rng, 1, 3600), M=M, C=C, groups=_groups(rng, C),
                        out=8 * _log(rng, 1, 640), full=full)
        w = work(case)
        if w["flops"] > (4e11 if case["dtype"] == "f32" else 2e12) or w["bytes"] > 4e8:
            continue
        if T * case["N"] * case.get("out", case.get("C", 0)) > 2e8:
            continue
        return case


def _frames(T, M):
    """M frames spread evenly over T with both ends among them (the first alone for M = 1)."""
    return [0] if M == 1 else [(2 * i * (T - 1) + M - 1) // (2 * (M - 1)) for i in range(M)]


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    rows = case["M"] * case["N"]
    if case["op"] == "norm":
        affine = {"none": 0, "one": 2, "frame": 2 * case["M"]}[case["affine"]]
        return {"bytes": (2 * rows + affine) * case["C"] * size, "flops": 10 * rows * case["C"]}
    if case["op"] == "norm8":
        C, n = case["C"], case["out"]
        return {"bytes": (rows * C + 2 * C + n + rows * n) * size + C * n + 4 * n, "flops": 2 * rows * C * n + 12 * rows * C}
    K, n = case["K"], case["out"]
    b = rows * n * (2 if case["residual"] else 1) + n + {"none": 0, "row": n, "frame": case["M"] * n}[case["gate"]]
    b = b * size + rows * (K + 4 if case["given"] else K * size) + K * n + 4 * n
    return {"bytes": b, "flops": 2 * rows * K * n}


def _rows8(x):
    """Rows of x (fp32) as whole numbers in fp32, and their scales (both quotients by way of 64 bits: dividing a tensor
    by a number, or a number by a tensor, may round twice)."""
    top = x.abs().amax(-1, keepdim=True)
    tiny = top < 2.0 ** -100
    q = (x * (127.0 / top.double()).float()).round()
    return q.masked_fill(tiny, 0.0), (top.double() / 127.0).float().masked_fill(tiny, 0.0)


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

    def features(rows, C):
        # channels of unlike size, a few much larger, around a mean of their own
        x = normal(rows, C)
        size = torch.exp(0.5 * torch.randn(C, generator=g, device="cuda"))
        size[::61] *= 6.0
        mean = torch.randn(C, generator=g, device="cuda")
        for part in x.split(max(1, (1 << 27) // C)):
            part.copy_(part.float() * size + mean)
        return x

    T, N, M = case["T"], case["N"], case["M"]
    st = {"case": case, "ids": np.array(_frames(T, M), dtype=np.int32)}
    rows = M * N
    C = case["K"] if case["op"] == "linear8" else case["C"]
    st["x"] = features(rows, C)
    if case["op"] != "linear8":
        affine = case.get("affine", "one")
        shape = (T, C) if affine == "frame" else (C,)
        st["w"] = None if affine == "none" else (1.0 + 0.2 * normal(*shape)).to(dt)
        st["b"] = None if affine == "none" else normal(*shape, scale=0.3)
    n = C
    if case["op"] != "norm":
        # the weight as a program holds it: 8-bit rows, a scale for each output feature
        n = case["out"]
        q, scale = _rows8(torch.randn((n, C), generator=g, device="cuda") / math.sqrt(C))
        st["wq"], st["ws"] = q.to(torch.int8), scale.reshape(-1).contiguous()
        st["bias"] = normal(n, scale=0.3)
        gate = case.get("gate", "none")
        st["gate"] = None if gate == "none" else normal(*((T, n) if gate == "frame" else (n,)), scale=0.5)
    out_rows = (T if case["full"] else M) * N
    st["residual"] = normal(out_rows, n) if case.get("residual") else None
    if case["op"] == "linear8" and case["given"]:
        q, scale = _rows8(st["x"].float())
        st["xq"], st["xs"] = q.to(torch.int8), scale.reshape(-1).contiguous()
    elif case["op"] != "norm":
        # where a program keeps the rows between its calls
        st["xq"] = torch.empty((rows, C), dtype=torch.int8, device="cuda")
        st["xs"] = torch.empty(rows, dtype=torch.float32, device="cuda")
    st["y"] = normal(out_rows, n) if case["full"] else torch.empty((out_rows, n), dtype=dt, device="cuda")
    if own:
        from paper_2606_06309_amd import binding as rf
        need = 16
        if case["op"] != "norm":
            need = max(need, rf.rf_frame_linear_i8_workspace(M, N, C, n, dt))
        if case["op"] != "linear8":
            need = max(need, rf.rf_frame_group_norm_workspace(M, N, C, case["groups"], dt, int8=case["op"] == "norm8",
                                                              frames_together=M if case.get("together") else 1))
        st["space"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    return st


def run(st):
    case = st["case"]
    if own:
        return _own(case, st)
    return {"norm": _norm, "linear8": _linear8, "norm8": _norm8}[case["op"]](case, st)


def _own(case, st):
    from paper_2606_06309_amd import binding as rf
    frames = dict(frame_ids=st["ids"], T=case["T"], rows_per_frame=case["N"])
    if case["op"] == "norm":
        return rf.rf_frame_group_norm(st["x"], case["groups"], st["w"], st["b"], eps=EPS, activation=case["act"],
                                      frames_together=case["M"] if case["together"] else 1, out_full=case["full"],
                                      out=st["y"], workspace=st["space"], **frames)
    if case["op"] == "norm8":
        rf.rf_frame_group_norm(st["x"], case["groups"], st["w"], st["b"], eps=EPS, out=st["xq"], out_scale=st["xs"],
                               workspace=st["space"], **frames)
        return rf.rf_frame_linear_i8(st["xq"], st["xs"], st["wq"], st["ws"], st["bias"], out_full=case["full"],
                                     out=st["y"], workspace=st["space"], **frames)
    if not case["given"]:
        rf.rf_frame_quantize(st["x"], out=st["xq"], out_scale=st["xs"])
    return rf.rf_frame_linear_i8(st["xq"], st["xs"], st["wq"], st["ws"], st["bias"], activation=case["act"],
                                 gate=st["gate"], residual=st["residual"], out_full=case["full"], out=st["y"],
                                 workspace=st["space"], **frames)


def _positions(case, device):
    """The position of every row of the listed frames among all frames' rows."""
    ids = torch.tensor(_frames(case["T"], case["M"]), device=device)
    return (ids[:, None] * case["N"] + torch.arange(case["N"], device=device)[None, :]).reshape(-1)


def _place(case, y, dst):
    """y's rows into dst, at their positions among all frames where the case says so."""
    if case["full"]:
        dst.index_copy_(0, _positions(case, y.device), y.to(dst.dtype))
    else:
        dst.copy_(y)
    return dst


def _activation(name, x):
    if name == "silu":
        return x / (1.0 + (-x).exp())
    if name == "gelu":
        return 0.5 * x * (1.0 + torch.erf(x * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * x * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x * x * x)))
    return x


def _of_frames(case, t):
    """A [T][C] tensor's rows of the listed frames, or a [C] one, against [M][N][C]."""
    if t.dim() == 1:
        return t
    return t[torch.tensor(_frames(case["T"], case["M"]), device=t.device)][:, None, :]


def _normed(case, st):
    """The normalised rows, [M][N][C] in 32 bits."""
    M, N, C, G = case["M"], case["N"], case["C"], case["groups"]
    shape = (1, M * N, G, C // G) if case.get("together") else (M, N, G, C // G)
    x = st["x"].float().view(shape)
    d = x - x.mean((1, 3), keepdim=True)
    y = (d * torch.rsqrt((d * d).mean((1, 3), keepdim=True) + EPS)).view(M, N, C)
    if st["w"] is not None:
        y = y * _of_frames(case, st["w"].float()) + _of_frames(case, st["b"].float())
    return _activation(case.get("act", "none"), y)


def _norm(case, st):
    return _place(case, _normed(case, st).view(-1, case["C"]), st["y"])


def _product(case, st, q, scale):
    """The 8-bit product's plain form, of rows as whole numbers in fp32."""
    y = torch.matmul(q, st["wq"].float().t()) * scale * st["ws"]
    y = _activation(case.get("act", "none"), y + st["bias"].float())
    if st["gate"] is not None:
        y = (y.view(case["M"], case["N"], -1) * _of_frames(case, st["gate"].float())).view(y.shape)
    if st["residual"] is not None:
        r = st["residual"].float()
        y = y + (r[_positions(case, y.device)] if case["full"] else r)
    return _place(case, y, st["y"])


def _linear8(case, st):
    if case["given"]:
        return _product(case, st, st["xq"].float(), st["xs"][:, None])
    return _product(case, st, *_rows8(st["x"].float()))


def _norm8(case, st):
    return _product(case, st, *_rows8(_normed(case, st).view(-1, case["C"])))


def exact(case, seed):
    st = prepare(case, seed)
    out = st["y"].double()
    frames, N = _frames(case["T"], case["M"]), case["N"]
    for m, f in enumerate(frames):
        if case["op"] == "linear8":
            part = st["x"][m * N:(m + 1) * N]
            y = _exact_product(case, st, part, f)
        else:
            part = _exact_norm(case, st, m, f)
            y = part if case["op"] == "norm" else _exact_product(case, st, part.float(), f)
        first = (f if case["full"] else m) * N
        if st["residual"] is not None:
            y = y + st["residual"][first:first + N].double()
        out[first:first + N] = y
    return out


def _exact_act(name, z):
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return z * torch.special.ndtr(z)
    if name == "gelu_tanh":
        return z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3))
    return z


def _exact_norm(case, st, m, f):
    """Frame f, the m-th listed: the moments of each channel, and of them those of each group."""
    N, C, G = case["N"], case["C"], case["groups"]
    if "moments" not in st:
        blocks = [st["x"][i * N:(i + 1) * N].double() for i in range(case["M"])] if case.get("together") else None
        if blocks is not None:
            mean = torch.stack([b.view(N, G, C // G).mean((0, 2)) for b in blocks]).mean(0)
            var = torch.stack([(b.view(N, G, C // G) - mean[:, None]).square().mean((0, 2)) for b in blocks]).mean(0)
            st["moments"] = mean, var
    x = st["x"][m * N:(m + 1) * N].double()
    if case.get("together"):
        mean, var = st["moments"]
    else:
        mean = x.mean(0).view(G, C // G).mean(1)
        var = (x - mean.repeat_interleave(C // G)).square().mean(0).view(G, C // G).mean(1)
    z = (x - mean.repeat_interleave(C // G)) / torch.sqrt(var + EPS).repeat_interleave(C // G)
    if st["w"] is not None:
        w, b = (t[f] if t.dim() == 2 else t for t in (st["w"].double(), st["b"].double()))
        z = z * w + b
    return _exact_act(case.get("act", "none"), z)


def _exact_product(case, st, part, f):
    """One frame's rows: rounded as they are defined to be (products of two fp32 numbers are whole in 64 bits), then
    multiplied."""
    top = part.double().abs().amax(1, keepdim=True)
    inverse = torch.where(top < 2.0 ** -100, torch.zeros_like(top), (127.0 / top).float().double())
    q = torch.round((part.double() * inverse).float().double())
    scale = torch.where(top < 2.0 ** -100, torch.zeros_like(top), (top / 127.0).float().double())
    z = torch.mm(q, st["wq"].double().t().contiguous()) * scale * st["ws"].double() + st["bias"].double()
    z = _exact_act(case.get("act", "none"), z)
    if st["gate"] is not None:
        z = z * (st["gate"][f] if st["gate"].dim() == 2 else st["gate"]).double()
    return z
