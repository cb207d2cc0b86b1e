"""Operators around the transformer block, each with its backward pass, and the cases they are measured on.

  rope         rotary positions for queries and keys: adjacent or split pairs, the whole head or its first
               part, the frequencies of long-context scalings; the backward pass is the rotation back
  norm         y = x_scale * x + h_scale * gate * (RMS(h) * w_post) and n = RMS(y) * w_pre: the norms
               behind one block and before the next, with the branch's gate and the residual scale
  xent         loss and log-sum-exp of the logits scale * X W^T against target tokens, and the gradients
               of X and W, without the logits ever being stored

`run` computes them in plain torch operations, or by the library's calls where `own` is true.
Sizes are those of this repository's workloads (hidden 4096 and 8192, 32 + 8 heads of 128, 16 + 4 heads of
64, 2048 to 16384 tokens) and generic ones around them.
"""
import math

import torch

own = False

IGNORE = -100
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
PARTS = dict(scaling="parts", factor=8.0, low=1.0, high=4.0, trained=8192, magnitude=1.0)
PLAIN = dict(scaling="none", factor=1.0, low=1.0, high=4.0, trained=0, magnitude=1.0)
LINEAR = dict(scaling="linear", factor=4.0, low=1.0, high=4.0, trained=0, magnitude=1.0)
STRONG = dict(scaling="parts", factor=32.0, low=1.0, high=32.0, trained=4096, magnitude=1.3466)


def listed():
    return [
        # one new token of each of 16 requests, far into their contexts: what counts is the launch
        dict(name="rope_decode", op="rope", dtype="bf16", B=16, S=1, H=32, Hkv=8, d=128, rot=128, layout="halves",
             theta=500000.0, far=100000, backward=False, fused=True, **PARTS),
        # queries and keys of a training sequence, read out of the fused QKV product
        dict(name="rope_16k", op="rope", dtype="bf16", B=1, S=16384, H=32, Hkv=8, d=128, rot=128, layout="interleaved",
             theta=500000.0, far=0, backward=False, fused=True, **PLAIN),
        # gradients of a small model's queries and keys, a part of the head rotated, ragged lengths
        dict(name="rope_back_part", op="rope", dtype="bf16", B=3, S=1999, H=16, Hkv=4, d=64, rot=32, layout="halves",
             theta=10000.0, far=5000, backward=True, fused=False, **STRONG),
        # residual stream of a few tokens being decoded
        dict(name="norm_decode", op="norm", dtype="bf16", rows=16, n=4096, gates=1, post=True, pre=True, x_scale=1.0,
             h_scale=0.25, backward=False),
        # the same of a long training sequence, without a gate
        dict(name="norm_16k", op="norm", dtype="bf16", rows=16384, n=4096, gates=0, post=True, pre=True, x_scale=1.0,
             h_scale=1.0, backward=False),
        # gradients of the wide layer, one gate a sequence
        dict(name="norm_back_8k", op="norm", dtype="bf16", rows=8192, n=8192, gates=4, post=True, pre=True, x_scale=1.0,
             h_scale=0.5, backward=True),
        # gradients in fp32 at sizes that are a multiple of nothing
        dict(name="norm_back_f32_odd", op="norm", dtype="f32", rows=1003, n=1001, gates=1, post=True, pre=True, x_scale=0.8,
             h_scale=1.0, backward=True),
        # scoring a handful of candidate tokens: the vocabulary's weights pass once
        dict(name="xent_score_16", op="xent", dtype="bf16", M=16, V=131072, K=4096, scale=1.0, ignored=0.0, dlse=False, train=False),
        # evaluation loss of a sequence
        dict(name="xent_eval_2k", op="xent", dtype="bf16", M=2048, V=131072, K=4096, scale=1.0, ignored=0.1, dlse=False, train=False),
        # loss and gradients of a small model in fp32, odd sizes
        dict(name="xent_train_f32", op="xent", dtype="f32", M=777, V=5003, K=513, scale=1.0, ignored=0.2, dlse=True, train=True),
        # loss and gradients of a short fine-tuning batch, vocabulary of no round size
        dict(name="xent_train_1k", op="xent", dtype="bf16", M=1000, V=50257, K=1024, scale=0.5, ignored=0.5, dlse=True, train=True),
        # loss and gradients of a training step
        dict(name="xent_train_8k", op="xent", dtype="bf16", M=8192, V=131072, K=4096, scale=1.0, ignored=0.05, dlse=False, train=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "norm", "norm", "xent", "xent"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "rope":
        d = rng.choice([64, 128, 128, 96, 80])
        H = rng.choice([8, 16, 32])
        B = rng.choice([1, 1, 2, 5, 16])
        S = max(1, _log_int(rng, 1, 16384 if dtype == "bf16" else 4096) // B)
        rot = rng.choice([d, d, d // 2, d // 4])
        return dict(op="rope", dtype=dtype, B=B, S=S, H=H, Hkv=rng.choice([H, H // 4]), d=d, rot=rot,
                    layout=rng.choice(["halves", "interleaved"]), theta=rng.choice([10000.0, 500000.0]),
                    far=rng.choice([0, 3000, 120000]), backward=rng.random() < 0.4, fused=rng.random() < 0.5,
                    **rng.choice([PLAIN, LINEAR, PARTS, STRONG]))
    if op == "norm":
        n = rng.choice([4096, 4096, 8192, 1024, 2816, 1000, 1001, _log_int(rng, 64, 8192)])
        gates = rng.choice([0, 1, 1, 3])
        rows = _log_int(rng, 1, 12000 if dtype == "bf16" else 6000)
        rows = max(1, rows // max(1, gates)) * max(1, gates)
        return dict(op="norm", dtype=dtype, rows=rows, n=n, gates=gates, post=rng.random() < 0.75, pre=rng.random() < 0.75,
                    x_scale=rng.choice([1.0, 1.0, 0.8]), h_scale=rng.choice([1.0, 0.5, 0.22]), backward=rng.random() < 0.6)
    train = rng.random() < 0.6
    if dtype == "f32":
        M, V, K = _log_int(rng, 1, 1024), _log_int(rng, 100, 8192), _log_int(rng, 64, 1024)
    else:
        M, V = _log_int(rng, 1, 6000), rng.choice([32000, 50257, 65536, 100003, 131072, _log_int(rng, 300, 131072)])
        K = rng.choice([512, 1024, 2048, 4096, 4096, 1000])
    return dict(op="xent", dtype=dtype, M=M, V=V, K=K, scale=rng.choice([1.0, 1.0, 0.5]), ignored=rng.choice([0.0, 0.1, 0.5]),
                dlse=rng.random() < 0.3, train=train)


def work(case):
    c, size = case, 2 if case["dtype"] == "bf16" else 4
    if c["op"] == "rope":
        heads = c["H"] + c["Hkv"]
        tokens = c["B"] * c["S"]
        return {"bytes": 2 * tokens * heads * c["d"] * size + 8 * tokens, "flops": 3 * tokens * heads * c["rot"]}
    if c["op"] == "norm":
        tensors = (4 + 2 * c["pre"] - (0 if c["post"] or c["gates"] else 1) if c["backward"] else 3 + c["pre"])
        vectors = (c["post"] + c["pre"] + c["gates"]) * c["n"]
        return {"bytes": tensors * c["rows"] * c["n"] * size + vectors * (size + (4 if c["backward"] else 0)),
                "flops": (30 if c["backward"] else 10) * c["rows"] * c["n"]}
    M, V, K = c["M"], c["V"], c["K"]
    once = (M + V) * K * size + 16 * M
    return {"bytes": (2 * once if c["train"] else once), "flops": (8 if c["train"] else 2) * M * V * K}


# ---------------------------------------------------------------- inputs
def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[c["dtype"]]
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=g)
    s = dict(case=c)
    if c["op"] == "rope":
        B, S, H, Hkv, d = c["B"], c["S"], c["H"], c["Hkv"], c["d"]
        if c["fused"]:      # queries, keys and values of a token side by side, as the QKV product leaves them
            qkv = normal(B, S, H + 2 * Hkv, d).to(dt)
            s["Q"], s["K"] = qkv[:, :, :H], qkv[:, :, H:H + Hkv]
        else:
            s["Q"], s["K"] = normal(B, S, H, d).to(dt), normal(B, S, Hkv, d).to(dt)
        first = torch.randint(0, c["far"] + 1, (B, 1), device="cuda", generator=g)
        s["positions"] = first + torch.arange(S, device="cuda")
    elif c["op"] == "norm":
        rows, n = c["rows"], c["n"]
        around_one = lambda *shape: (1.0 + 0.1 * normal(*shape)).to(dt)
        s["w_post"] = around_one(n) if c["post"] else None
        s["w_pre"] = around_one(n) if c["pre"] else None
        s["gate"] = (0.5 + 0.5 * normal(c["gates"], n)).to(dt) if c["gates"] else None
        s["h"] = (0.7 * normal(rows, n)).to(dt)
        if c["backward"]:
            s["y"], s["dy"] = (2.0 * normal(rows, n)).to(dt), normal(rows, n).to(dt)
            s["dn"] = normal(rows, n).to(dt) if c["pre"] else None
        else:
            s["x"] = (2.0 * normal(rows, n)).to(dt)
    else:
        M, V, K = c["M"], c["V"], c["K"]
        W = (0.02 * normal(V, K)).to(dt)
        t = torch.randint(0, V, (M,), device="cuda", generator=g)
        # hidden states lean towards their target, as a trained model's do
        s["X"] = (normal(M, K) + 3.0 / (0.0004 * K) * W[t].float()).to(dt)
        s["W"] = W
        s["targets"] = torch.where(torch.rand(M, device="cuda", generator=g) < c["ignored"], torch.full_like(t, IGNORE), t)
        if c["train"]:
            kept = (s["targets"] != IGNORE).sum().clamp(min=1)
            s["dloss"] = torch.ones(M, device="cuda") / kept
            s["dlse"] = 0.01 * torch.rand(M, device="cuda", generator=g) / kept if c["dlse"] else None
    return s


# ---------------------------------------------------------------- one pass
def run(state):
    c = state["case"]
    if own:
        return {"rope": _rope_own, "norm": _norm_own, "xent": _xent_own}[c["op"]](state, c)
    return {"rope": _rope_plain, "norm": _norm_plain, "xent": _xent_plain}[c["op"]](state, c)


def _rope_own(s, c):
    from paper_2410_07531_amd import binding as rov
    cfg = rov.make_rope_cfg(c["rot"], c["theta"],
                            layout=rov.ROPE_HALVES if c["layout"] == "halves" else rov.ROPE_INTERLEAVED,
                            scaling={"none": rov.ROPE_SCALE_NONE, "linear": rov.ROPE_SCALE_LINEAR, "parts": rov.ROPE_SCALE_PARTS}[c["scaling"]],
                            factor=c["factor"], turns_low=c["low"], turns_high=c["high"], trained_len=c["trained"], magnitude=c["magnitude"])
    return rov.rope(cfg, s["Q"], s["K"], positions=s["positions"], backward=c["backward"])


def _norm_own(s, c):
    from paper_2410_07531_amd import binding as rov
    kw = dict(w_pre=s["w_pre"], w_post=s["w_post"], gate=s["gate"], x_scale=c["x_scale"], h_scale=c["h_scale"], eps=1e-5)
    if c["backward"]:
        return rov.norm_residual_bwd(s["y"], s["h"], s["dy"], s["dn"], **kw)
    return rov.norm_residual(s["x"], s["h"], **kw)


def _xent_own(s, c):
    from paper_2410_07531_amd import binding as rov
    loss, lse = rov.linear_xent(s["X"], s["W"], s["targets"], scale=c["scale"], ignore_index=IGNORE)
    if not c["train"]:
        return loss, lse
    dX, dW = rov.linear_xent_bwd(s["X"], s["W"], s["targets"], lse, s["dloss"], s["dlse"], scale=c["scale"], ignore_index=IGNORE)
    return loss, lse, dX, dW


# ---------------------------------------------------------------- plain forms
def _frequencies(c):
    f = c["theta"] ** (-torch.arange(0, c["rot"], 2, device="cuda", dtype=torch.float64) / c["rot"])
    if c["scaling"] == "linear":
        f = f / c["factor"]
    if c["scaling"] == "parts":
        turns = c["trained"] * f / (2.0 * math.pi)
        keep = ((turns - c["low"]) / (c["high"] - c["low"])).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / c["factor"])
    return f


def _rope_plain(s, c):
    angle = s["positions"].double()[:, :, None] * _frequencies(c)        # [B, S, rot / 2]
    cos = (c["magnitude"] * torch.cos(angle)).float()[:, :, None]
    sin = (c["magnitude"] * torch.sin(angle)).float()[:, :, None]
    if c["backward"]:
        sin = -sin
    rot = c["rot"]

    def turn(x):
        v = x.float()
        out = v.clone()
        if c["layout"] == "halves":
            a, b = v[..., :rot // 2], v[..., rot // 2:rot]
            out[..., :rot // 2], out[..., rot // 2:rot] = a * cos - b * sin, a * sin + b * cos
        else:
            a, b = v[..., 0:rot:2], v[..., 1:rot:2]
            out[..., 0:rot:2], out[..., 1:rot:2] = a * cos - b * sin, a * sin + b * cos
        return out.to(x.dtype)

    return turn(s["Q"]), turn(s["K"])


def _norm_plain(s, c):
    n, eps, dt = c["n"], 1e-5, s["h"].dtype
    groups = max(1, c["gates"])
    vec = lambda v: 1.0 if v is None else v.float()
    gate = 1.0 if s["gate"] is None else s["gate"].float()[:, None, :]
    by_group = lambda v: v.reshape(groups, -1, n)
    h = s["h"].float()
    inv_h = torch.rsqrt((h * h).mean(1, keepdim=True) + eps) if c["post"] else torch.ones_like(h[:, :1])
    unit = h * inv_h
    if not c["backward"]:
        branch = (by_group(unit * vec(s["w_post"])) * gate).reshape(h.shape)
        y = c["x_scale"] * s["x"].float() + c["h_scale"] * branch
        if not c["pre"]:
            return y.to(dt), None
        return y.to(dt), (y * torch.rsqrt((y * y).mean(1, keepdim=True) + eps) * s["w_pre"].float()).to(dt)
    gy, dw_pre, dw_post, dgate = s["dy"].float(), None, None, None
    if c["pre"]:
        y, dn = s["y"].float(), s["dn"].float()
        inv_y = torch.rsqrt((y * y).mean(1, keepdim=True) + eps)
        t = dn * s["w_pre"].float()
        gy = gy + inv_y * t - y * inv_y ** 3 * (y * t).mean(1, keepdim=True)
        dw_pre = (dn * y * inv_y).sum(0)
    q = c["h_scale"] * (by_group(gy) * gate).reshape(h.shape)
    t = q * vec(s["w_post"])
    dh = t
    if c["post"]:
        dh = inv_h * t - h * inv_h ** 3 * (h * t).mean(1, keepdim=True)
        dw_post = (q * unit).sum(0)
    if c["gates"]:
        dgate = by_group(c["h_scale"] * gy * unit * vec(s["w_post"])).sum(1)
    return (c["x_scale"] * gy).to(dt), dh.to(dt), dw_pre, dw_post, dgate


def _xent_plain(s, c):
    X, W, t = s["X"].float(), s["W"].float(), s["targets"]
    z = c["scale"] * (X @ W.t())
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    valid = t != IGNORE
    at = torch.where(valid, t, torch.zeros_like(t))[:, None]
    loss = torch.where(valid, lse - z.gather(1, at)[:, 0], torch.zeros_like(lse))
    if not c["train"]:
        return loss, lse
    up = s["dloss"] if s["dlse"] is None else s["dloss"] + s["dlse"]
    G = e / total * (up * valid)[:, None]
    G.scatter_add_(1, at, -(s["dloss"] * valid)[:, None])
    G = c["scale"] * G
    return loss, lse, (G @ W).to(s["X"].dtype), (G.t() @ X).to(s["W"].dtype)


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    c, s = dict(case), prepare(case, seed)
    return {"rope": _rope_exact, "norm": _norm_exact, "xent": _xent_exact}[c["op"]](s, c)


def _rope_exact(s, c):
    rot, half = c["rot"], c["rot"] // 2
    f = []
    for p in range(half):
        w = math.exp(-2.0 * p / rot * math.log(c["theta"]))
        if c["scaling"] == "linear":
            w /= c["factor"]
        elif c["scaling"] == "parts":
            r = (c["trained"] * w / (2.0 * math.pi) - c["low"]) / (c["high"] - c["low"])
            r = min(1.0, max(0.0, r))
            w = r * w + (1.0 - r) * w / c["factor"]
        f.append(w)
    angle = s["positions"][:, :, None].double() * torch.tensor(f, dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.full_like(angle, c["magnitude"]), -angle if c["backward"] else angle)[:, :, None]

    def one(x):
        v, rest = x[..., :rot].double(), x[..., rot:].double()
        pairs = v.unflatten(-1, (2, half)).transpose(-1, -2) if c["layout"] == "halves" else v.unflatten(-1, (half, 2))
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        z = (z.transpose(-1, -2) if c["layout"] == "halves" else z).flatten(-2)
        return torch.cat([z, rest], -1)

    return one(s["Q"]), one(s["K"])


def _norm_exact(s, c):
    # the backward pass by automatic differentiation of the definition
    leaf = lambda v: None if v is None else v.double().requires_grad_(c["backward"])
    h, w_post, w_pre, gate = leaf(s["h"]), leaf(s["w_post"]), leaf(s["w_pre"]), leaf(s["gate"])
    rms = lambda v: v / torch.sqrt(torch.mean(v ** 2, -1, keepdim=True) + 1e-5)
    branch = h if w_post is None else rms(h) * w_post
    if gate is not None:
        branch = branch * gate.repeat_interleave(c["rows"] // c["gates"], 0)
    branch = c["h_scale"] * branch
    if not c["backward"]:
        y = c["x_scale"] * s["x"].double() + branch
        return y, None if w_pre is None else rms(y) * w_pre
    # y is given, rounded as the forward pass left it: the stream that x came in by makes up the rest
    x = ((s["y"].double() - branch.detach()) / c["x_scale"]).requires_grad_(True)
    y = c["x_scale"] * x + branch
    total = (y * s["dy"].double()).sum()
    if w_pre is not None:
        total = total + (rms(y) * w_pre * s["dn"].double()).sum()
    total.backward()
    grad = lambda v: None if v is None else v.grad
    return x.grad, h.grad, grad(w_pre), grad(w_post), grad(gate)


def _xent_exact(s, c):
    W = s["W"].double()
    loss, lse, dX, dW = [], [], [], torch.zeros_like(W)
    for r in range(0, c["M"], 2048):
        x, t = s["X"][r:r + 2048].double(), s["targets"][r:r + 2048]
        z = (x @ W.T) * c["scale"]
        total = torch.logsumexp(z, 1)
        rows = torch.arange(len(t), device=t.device)
        kept = t >= 0
        picked = z[rows, t.clamp(min=0)]
        lse.append(total)
        loss.append((total - picked) * kept)
        if c["train"]:
            a = s["dloss"][r:r + 2048].double() * kept
            b = a if s["dlse"] is None else a + s["dlse"][r:r + 2048].double() * kept
            z = torch.softmax(z, 1) * b[:, None]
            z[rows, t.clamp(min=0)] -= a
            z *= c["scale"]
            dX.append(z @ W)
            dW += z.T @ x
    if not c["train"]:
        return torch.cat(loss), torch.cat(lse)
    return torch.cat(loss), torch.cat(lse), torch.cat(dX), dW
