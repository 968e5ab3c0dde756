"""Group normalisation with an activation and 8-bit activation checkpoints, as cases that can be timed and compared one by one.

Kinds of cases
  fwd         pt_gn_act_fwd: y = act(gamma * xhat + beta + residual), statistics per image and group of channels
  bwd         pt_gn_act_bwd: the gradients, from the saved bf16 input and its statistics
  bwd8        pt_gn_act_bwd_packed: the same from the input's 8-bit checkpoint; the activation comes back too, for the weight
              gradient of the convolution that read it
  checkpoint  pt_act_pack, then pt_act_unpack: an activation into 8 bits and back
  layer8      a training step's share of one layer: the forward pass that leaves the checkpoint, the backward pass that reads it

Tensors are NHWC bf16 with a channel pitch that is a multiple of 16, as the convolutions read and write them; parameters and
statistics are fp32. A checkpoint holds one int8 code per value and one byte per block of 32 consecutive channels of a pixel: the
block's scale is 2^(byte - 127), the smallest power of two, of 2^-127 .. 2^121, that brings its values into [-127, 127]. Byte 255: the block
stands for NaN.
"""
import math

import torch

own = False
EPS = 1e-5
NONE, RELU, SILU = 0, 1, 2


# ------------------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # the smallest call a user makes: a CIFAR-sized layer with ragged channels and groups, small batch; latency
        dict(name="fwd tiny 16x16x27 b8", kind="fwd", N=8, H=16, C=27, G=4, act=RELU, residual=False),
        # the end of a pruned ImageNet bottleneck: wide, uneven groups, the residual add
        dict(name="fwd 28x28x371 b64 res", kind="fwd", N=64, H=28, C=371, G=32, act=RELU, residual=True),
        # few large images, where images alone do not fill the device: what group norm is for
        dict(name="fwd 112x112x64 b2 silu", kind="fwd", N=2, H=112, C=64, G=16, act=SILU, residual=False),
        # the last stage of the CIFAR ResNet-32: many small images
        dict(name="bwd 8x8x64 b128", kind="bwd", N=128, H=8, C=64, G=8, act=RELU, residual=False),
        # the end of the pruned bottleneck again, and the dense stage-1 output
        dict(name="bwd 28x28x371 b64 res", kind="bwd", N=64, H=28, C=371, G=32, act=RELU, residual=True),
        dict(name="bwd 56x56x256 b64 silu", kind="bwd", N=64, H=56, C=256, G=32, act=SILU, residual=False),
        # the activations between two layers saved in 8 bits: a small pruned one, the largest one
        dict(name="checkpoint 8x8x41 b128", kind="checkpoint", N=128, H=8, C=41),
        dict(name="checkpoint 56x56x256 b64", kind="checkpoint", N=64, H=56, C=256),
        # the backward pass from checkpoints: the wide end of a pruned stage-3 bottleneck
        dict(name="bwd8 14x14x931 b64 res", kind="bwd8", N=64, H=14, C=931, G=32, act=RELU, residual=True),
        # both directions of a layer with its checkpoint: the CIFAR ResNet-32's first stage; the dense ImageNet stage-1
        # output, the largest map behind the stem, larger than the L2 cache
        dict(name="layer8 32x32x16 b128", kind="layer8", N=128, H=32, C=16, G=4, act=SILU, residual=False),
        dict(name="layer8 56x56x256 b64", kind="layer8", N=64, H=56, C=256, G=32, act=SILU, residual=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _one(rng):
    kind = rng.choice(["fwd", "fwd", "bwd", "bwd", "bwd8", "checkpoint", "layer8"])
    C = _log(rng, 8, 2048)
    H = rng.choice([1, 4, 7, 8, 14, 16, 28, 32, 56, 112, rng.randint(1, 64), rng.randint(1, 64)])
    if C * H * H < 64:
        H = 8
    c = dict(kind=kind, N=_log(rng, 1, 256), H=H, C=C)
    if kind != "checkpoint":
        # (groups of a few values have no gradient to speak of: the statistics take it all)
        c["G"] = min(C, C * H * H // 64, rng.choice([1, 2, 4, 8, 16, 32, 32, 64, rng.randint(1, 64)]))
        # a layer of both passes is smooth: its ReLU would be decided by the last bits of the statistics
        c["act"] = SILU if kind == "layer8" else rng.choice([NONE, RELU, RELU, SILU])
        c["residual"] = rng.random() < 0.4
    return c


def draw(rng):
    """One more case of the ranges above; one that would cost more than the largest listed one is drawn again."""
    most = max(work(c)["bytes"] for c in listed())
    while True:
        c = _one(rng)
        if work(c)["bytes"] <= most:
            return c


# ------------------------------------------------------------------------------------------------ prepare
def _pitch(C):
    return (C + 15) // 16 * 16


def _begin(C, G):
    """First channel of every group, and C: as equal as whole channels allow."""
    return [g * C // G for g in range(G + 1)]


def _member(begin, device):
    """[C][G]: 1 where the channel belongs to the group."""
    b = torch.tensor(begin, device=device)
    c = torch.arange(begin[-1], device=device).unsqueeze(1)
    return ((c >= b[:-1]) & (c < b[1:])).double()


def _quantise(x):
    """[..., C] -> (codes int8 [..., C], scale bytes uint8 [..., ceil(C / 32)])."""
    C = x.shape[-1]
    nb = (C + 31) // 32
    f = torch.nn.functional.pad(x.float(), (0, nb * 32 - C)).unflatten(-1, (nb, 32))
    amax = f.abs().amax(-1)
    bad = ~torch.isfinite(f).all(-1)
    m, k = torch.frexp(torch.where(bad, torch.zeros_like(amax), amax))   # amax = m * 2^k, m in [0.5, 1): m * 128 rounds to 128 from 127.5 on
    e = torch.where(m * 128 >= 127.5, k - 6, k - 7).clamp_(min=-127, max=121)
    e = torch.where(amax == 0, torch.full_like(e, -127), e)
    # (2^-e in two factors: one alone may be too large for fp32)
    q = torch.ldexp(torch.ldexp(f, (-e // 2).unsqueeze(-1)), (-e - (-e // 2)).unsqueeze(-1)).round_().clamp_(min=-127, max=127)
    q = torch.where(bad.unsqueeze(-1), torch.zeros_like(q), q)
    return q.flatten(-2)[..., :C].to(torch.int8), torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)


def _dequantise(codes, scales):
    """The fp32 values that codes and scale bytes stand for."""
    C = codes.shape[-1]
    s = scales.double()
    s = torch.where(s == 255, torch.full_like(s, float("nan")), torch.exp2(s - 127))
    return (codes.double() * s.repeat_interleave(32, -1)[..., :C]).float()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    N, H, C = case["N"], case["H"], case["C"]
    ld, shape = _pitch(C), (N, H, H, _pitch(C))
    s = dict(case=case, ld=ld)
    # a convolution's output: channels of different strength and offset (an activation behind a ReLU where it is saved by itself)
    strength = torch.rand(ld, generator=g, device="cuda") * 1.5 + 0.25
    x = torch.randn(shape, generator=g, device="cuda") * strength + (torch.rand(ld, generator=g, device="cuda") - 0.25)
    s["x"] = (x.clamp_(min=0) if case["kind"] == "checkpoint" else x).to(torch.bfloat16)
    if case["kind"] == "checkpoint":
        return s
    s["begin"] = _begin(C, case["G"])
    s["gamma"] = torch.rand(C, generator=g, device="cuda") + 0.5
    s["beta"] = torch.rand(C, generator=g, device="cuda") - 0.5
    s["res"] = torch.randn(shape, generator=g, device="cuda").clamp_(min=0).to(torch.bfloat16) if case["residual"] else None
    if case["kind"] != "fwd":
        s["dy"] = (torch.randn(shape, generator=g, device="cuda") * 2.0 ** -6).to(torch.bfloat16)
    if case["kind"] in ("bwd", "bwd8"):            # what the forward pass saved
        f = s["x"][..., :C]
        mem = _member(s["begin"], f.device)
        m = mem.sum(0) * H * H
        mean = f.sum((1, 2), dtype=torch.float64) @ mem / m
        d = f.float() - (mean @ mem.T).float()[:, None, None]
        var = d.square_().sum((1, 2), dtype=torch.float64) @ mem / m
        s["mean"], s["rstd"] = mean.float(), (var + EPS).rsqrt().float()
    if case["kind"] == "bwd8":
        codes, scales = _quantise(s["x"][..., :C])
        s["codes"] = torch.zeros((N, H, H, (C + 7) // 8 * 8), dtype=torch.int8, device="cuda")
        s["codes"][..., :C] = codes
        s["scales"] = torch.zeros((scales.numel() + 15) // 16 * 16, dtype=torch.uint8, device="cuda")
        s["scales"][:scales.numel()] = scales.flatten()
        s["nb"] = scales.shape[-1]
        del s["x"]
    return s


# ------------------------------------------------------------------------------------------------ the plain forms
def _spread(v, mem):
    """[N][G] -> [N][1][1][C]."""
    return (v.double() @ mem.T)[:, None, None]


def _plain_fwd(s):
    c = s["case"]
    C = c["C"]
    x = s["x"][..., :C].float()
    mem = _member(s["begin"], x.device)
    m = mem.sum(0) * x.shape[1] * x.shape[2]
    mean = x.sum((1, 2), dtype=torch.float64) @ mem / m
    d = x - _spread(mean, mem).float()
    var = d.square().sum((1, 2), dtype=torch.float64) @ mem / m
    rstd = (var + EPS).rsqrt()
    z = d * _spread(rstd, mem).float() * s["gamma"] + s["beta"]
    if s["res"] is not None:
        z = z + s["res"][..., :C].float()
    return _act(z, c["act"]).to(torch.bfloat16), mean.float(), rstd.float()


def _act(z, act):
    return z.clamp(min=0) if act == RELU else z / (1 + torch.exp(-z)) if act == SILU else z


def _plain_bwd(s, x, mean, rstd):
    c = s["case"]
    C, act = c["C"], c["act"]
    mem = _member(s["begin"], x.device)
    m = mem.sum(0) * x.shape[1] * x.shape[2]
    # on which side of 0 a value lies is decided in 64 bits
    wide = torch.float64 if act == RELU else torch.float32
    r = _spread(rstd, mem).float()
    xhat = (x.to(wide) - _spread(mean, mem).to(wide)) * r
    z = xhat * s["gamma"] + s["beta"]
    if s["res"] is not None:
        z = z + s["res"][..., :C]
    xhat = xhat.float()
    dy = s["dy"][..., :C].float()
    if act == RELU:
        dz = dy * (z > 0)
    elif act == SILU:
        sig = 1 / (1 + torch.exp(-z))
        dz = dy * sig * (1 + z * (1 - sig))
    else:
        dz = dy
    sdz = dz.sum((1, 2), dtype=torch.float64)
    sdx = (dz * xhat).sum((1, 2), dtype=torch.float64)
    a = _spread((sdz * s["gamma"]) @ mem / m, mem).float()
    b = _spread((sdx * s["gamma"]) @ mem / m, mem).float()
    dx = r * (dz * s["gamma"] - a - xhat * b)
    out = {"dx": dx.to(torch.bfloat16), "dgamma": sdx.sum(0).float(), "dbeta": sdz.sum(0).float()}
    if s["res"] is not None:
        out["dresidual"] = dz.to(torch.bfloat16)
    return out, _act(z.float(), act).to(torch.bfloat16)


def _run_plain(s):
    c = s["case"]
    C = c["C"]
    if c["kind"] == "fwd":
        return dict(zip(("y", "mean", "rstd"), _plain_fwd(s)))
    if c["kind"] == "bwd":
        return _plain_bwd(s, s["x"][..., :C].float(), s["mean"], s["rstd"])[0]
    if c["kind"] == "bwd8":
        n = s["codes"].shape[:3] + (s["nb"],)
        out, y = _plain_bwd(s, _dequantise(s["codes"][..., :C], s["scales"][:math.prod(n)].view(n)), s["mean"], s["rstd"])
        return dict(out, y=y)
    x = _dequantise(*_quantise(s["x"][..., :C]))
    if c["kind"] == "checkpoint":
        return x.to(torch.bfloat16)
    y, mean, rstd = _plain_fwd(s)
    out, again = _plain_bwd(s, x, mean, rstd)
    return dict(out, y=y, mean=mean, rstd=rstd, y_again=again)


# ------------------------------------------------------------------------------------------------ the framework's calls
_CTX = []


def _plan(s):
    """What a program that trains with these calls keeps: the context, descriptors, output buffers, workspace."""
    from paper_1901_09290_b200 import binding as B
    if not _CTX:
        _CTX.append(B.Context(0))
    c = s["case"]
    N, H, C = c["N"], c["H"], c["C"]
    p = dict(B=B, ctx=_CTX[0])
    bf = lambda: torch.empty((N, H, H, s["ld"]), dtype=torch.bfloat16, device="cuda")
    if c["kind"] == "checkpoint":
        p["d"] = B.make_pack_desc(N * H * H, C, s["ld"])
        p["codes"], p["scales"] = B.checkpoint_buffers(N * H * H, C)
        p["y"] = bf()
        return p
    p["d"] = d = B.make_gn_desc(N, H, H, C, c["G"], s["ld"], EPS, c["act"], group_begin=s["begin"])
    if c["kind"] in ("fwd", "layer8"):
        p["y"] = bf()
        p["mean"], p["rstd"] = (torch.empty((N, c["G"]), device="cuda") for _ in range(2))
    if c["kind"] == "layer8":
        p["codes"], p["scales"] = B.checkpoint_buffers(N * H * H, C)
    if c["kind"] in ("bwd8", "layer8"):
        p["again"] = bf()
    if c["kind"] != "fwd":
        p["dx"], p["dres"] = bf(), bf() if c["residual"] else None
        p["dgamma"], p["dbeta"] = (torch.empty(C, device="cuda") for _ in range(2))
        p["ws"] = torch.empty(B.pt_gn_workspace_bytes(p["ctx"], d), dtype=torch.uint8, device="cuda")
    return p


def _run_own(s):
    if "plan" not in s:
        s["plan"] = _plan(s)
    p, kind = s["plan"], s["case"]["kind"]
    B, ctx, d, C = p["B"], p["ctx"], p["d"], s["case"]["C"]
    if kind == "checkpoint":
        B.pt_act_pack(ctx, d, s["x"], p["codes"], p["scales"])
        B.pt_act_unpack(ctx, d, p["codes"], p["scales"], p["y"])
        return p["y"][..., :C]
    if kind == "fwd":
        B.pt_gn_act_fwd(ctx, d, s["x"], s["res"], s["gamma"], s["beta"], p["mean"], p["rstd"], p["y"])
        return {"y": p["y"][..., :C], "mean": p["mean"], "rstd": p["rstd"]}
    if kind == "bwd":
        B.pt_gn_act_bwd(ctx, d, s["x"], s["res"], s["dy"], s["gamma"], s["beta"], s["mean"], s["rstd"], p["dx"], p["dres"], p["dgamma"],
                        p["dbeta"], p["ws"])
    elif kind == "bwd8":
        B.pt_gn_act_bwd_packed(ctx, d, s["codes"], s["scales"], s["res"], s["dy"], s["gamma"], s["beta"], s["mean"], s["rstd"], p["dx"],
                               p["dres"], p["dgamma"], p["dbeta"], p["again"], p["ws"])
    else:
        B.pt_gn_act_fwd(ctx, d, s["x"], s["res"], s["gamma"], s["beta"], p["mean"], p["rstd"], p["y"], p["codes"], p["scales"])
        B.pt_gn_act_bwd_packed(ctx, d, p["codes"], p["scales"], s["res"], s["dy"], s["gamma"], s["beta"], p["mean"], p["rstd"], p["dx"],
                               p["dres"], p["dgamma"], p["dbeta"], p["again"], p["ws"])
    out = {"dx": p["dx"][..., :C], "dgamma": p["dgamma"], "dbeta": p["dbeta"]}
    if p["dres"] is not None:
        out["dresidual"] = p["dres"][..., :C]
    if kind == "bwd8":
        out["y"] = p["again"][..., :C]
    if kind == "layer8":
        out.update(y=p["y"][..., :C], mean=p["mean"], rstd=p["rstd"], y_again=p["again"][..., :C])
    return out


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------------ work and exact values
def work(case):
    N, H, C, kind = case["N"], case["H"], case["C"], case["kind"]
    e = float(N * H * H * C)
    code = e + N * H * H * ((C + 31) // 32)
    if kind == "checkpoint":
        return {"bytes": 2 * (2 * e + code), "flops": 4 * e}
    res = 2 * e if case["residual"] else 0.0
    stats = 8.0 * N * case["G"] + 8.0 * C
    fwd = 4 * e + res + stats
    bwd = {"bwd": 2 * e, "bwd8": code + 2 * e, "layer8": code + 2 * e}.get(kind, 0) + 4 * e + 2 * res + stats + 8.0 * C
    if kind == "fwd":
        return {"bytes": fwd, "flops": 10 * e}
    if kind == "layer8":
        return {"bytes": fwd + code + bwd, "flops": 30 * e}
    return {"bytes": bwd, "flops": 20 * e}


def exact(case, seed):
    s = prepare(case, seed)
    kind, C, hw = case["kind"], case["C"], case["H"] ** 2

    def stored(v):
        """The values an 8-bit checkpoint of v [..., C] holds, block by block: the step is the least power of two that keeps the codes within 127."""
        v = v.double()
        out = torch.empty_like(v)
        for b in range(0, v.shape[-1], 32):
            blk = v[..., b:b + 32]
            top = blk.abs().amax(-1, keepdim=True)
            step = torch.exp2(torch.ceil(torch.log2(top.clamp(min=1e-300) / 127)))
            step = torch.where(torch.round(top / (step / 2)) <= 127, step / 2, step).clamp(min=2.0 ** -127, max=2.0 ** 121)
            out[..., b:b + 32] = torch.round(blk / step).clamp(min=-127, max=127) * step
        return out

    if kind == "checkpoint":
        return stored(s["x"][..., :C])
    gamma, beta = s["gamma"].double(), s["beta"].double()
    res = s["res"][..., :C].double() if s["res"] is not None else None

    def act(z):
        return torch.where(z > 0, z, torch.zeros_like(z)) if case["act"] == RELU else z * torch.sigmoid(z) if case["act"] == SILU else z

    out = {}
    groups = list(zip(s["begin"][:-1], s["begin"][1:]))
    if kind in ("fwd", "layer8"):
        x = s["x"][..., :C].double()
        out["y"], out["mean"], out["rstd"] = torch.empty_like(x), [], []
        for b, e in groups:
            part = x[..., b:e]
            mu = part.mean((1, 2, 3))
            r = 1 / torch.sqrt((part - mu[:, None, None, None]).pow(2).mean((1, 2, 3)) + EPS)
            z = (part - mu[:, None, None, None]) * r[:, None, None, None] * gamma[b:e] + beta[b:e]
            out["y"][..., b:e] = act(z if res is None else z + res[..., b:e])
            out["mean"].append(mu)
            out["rstd"].append(r)
        out["mean"], out["rstd"] = torch.stack(out["mean"], 1), torch.stack(out["rstd"], 1)
        if kind == "fwd":
            return out
        mean, rstd = out["mean"], out["rstd"]
        x = stored(s["x"][..., :C])
    else:
        mean, rstd = s["mean"].double(), s["rstd"].double()
        if kind == "bwd":
            x = s["x"][..., :C].double()
        else:
            q = s["codes"][..., :C].double()
            byte = s["scales"][:q[..., 0].numel() * s["nb"]].view(*q.shape[:3], s["nb"]).double()
            x = torch.cat([q[..., 32 * b:32 * b + 32] * torch.exp2(byte[..., b:b + 1] - 127) for b in range(s["nb"])], -1)
    dy = s["dy"][..., :C].double()
    dx, dres, again = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    dgamma, dbeta = torch.empty(C, dtype=torch.float64, device=x.device), torch.empty(C, dtype=torch.float64, device=x.device)
    for g, (b, e) in enumerate(groups):
        r = rstd[:, g, None, None, None]
        xhat = (x[..., b:e] - mean[:, g, None, None, None]) * r
        z = xhat * gamma[b:e] + beta[b:e]
        z = z if res is None else z + res[..., b:e]
        sig = torch.sigmoid(z)
        slope = (z > 0).double() if case["act"] == RELU else sig + z * sig * (1 - sig) if case["act"] == SILU else torch.ones_like(z)
        dz = dy[..., b:e] * slope
        dbeta[b:e], dgamma[b:e] = dz.sum((0, 1, 2)), (dz * xhat).sum((0, 1, 2))
        w = dz * gamma[b:e]
        m = float(hw * (e - b))
        first, second = w.sum((1, 2, 3), keepdim=True) / m, (w * xhat).sum((1, 2, 3), keepdim=True) / m
        dx[..., b:e], dres[..., b:e], again[..., b:e] = r * (w - first - second * xhat), dz, act(z)
    out.update(dx=dx, dgamma=dgamma, dbeta=dbeta)
    if res is not None:
        out["dresidual"] = dres
    if kind == "bwd8":
        out["y"] = again
    if kind == "layer8":
        out["y_again"] = again
    return out
