"""Rotary positions against the formula in 64 bits.

Tolerance of an element m * (a cos t - b sin t): the sine's and cosine's error (angle reduced in double, rounded to
fp32: pi * 2^-24; sincosf about 2^-24) times |a| + |b|, with the fp32 products and sum together below 2^-21 * m (|a| + |b|);
bf16 results are off by another half step, 2^-8 of the value.
"""
import math

import pytest
import torch

from paper_2410_07531_amd import binding as rov

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
PARTS = dict(scaling=rov.ROPE_SCALE_PARTS, factor=8.0, turns_low=1.0, turns_high=4.0, trained_len=8192, magnitude=1.25)
LINEAR = dict(scaling=rov.ROPE_SCALE_LINEAR, factor=4.0)


def _freq(c):
    out = []
    for p in range(c["rot"] // 2):
        f = c["theta"] ** (-2.0 * p / c["rot"])
        if c.get("scaling") == rov.ROPE_SCALE_LINEAR:
            f /= c["factor"]
        if c.get("scaling") == rov.ROPE_SCALE_PARTS:
            r = c["trained_len"] * f / (2 * math.pi)
            k = min(1.0, max(0.0, (r - c["turns_low"]) / (c["turns_high"] - c["turns_low"])))
            f *= k + (1 - k) / c["factor"]
        out.append(f)
    return torch.tensor(out, dtype=torch.float64)


def reference(x, pos, c, backward=False):
    """(result, |a| + |b| of each element's pair) in float64 on the CPU; pos [B, S] or None."""
    x = x.double().cpu()
    B, S, _, d = x.shape
    pos = torch.arange(S)[None].expand(B, S) if pos is None else pos.cpu().reshape(-1, S).expand(B, S)
    t = pos.double()[:, :, None, None] * _freq(c)
    m = torch.tensor(c.get("magnitude", 1.0), dtype=torch.float32).double()
    cos, sin = m * torch.cos(t), m * torch.sin(-t if backward else t)
    rot, half = c["rot"], c["rot"] // 2
    ia = torch.arange(half) if c["layout"] == rov.ROPE_HALVES else 2 * torch.arange(half)
    ib = ia + half if c["layout"] == rov.ROPE_HALVES else ia + 1
    a, b = x[..., ia], x[..., ib]
    out, mag = x.clone(), torch.zeros_like(x)
    out[..., ia], out[..., ib] = a * cos - b * sin, a * sin + b * cos
    mag[..., ia] = mag[..., ib] = m * (a.abs() + b.abs())
    return out, mag


def close(got, want, mag, dtype):
    err = (got.double().cpu() - want).abs()
    tol = 2.0 ** -21 * mag + (2.0 ** -8 * want.abs() if dtype == "bf16" else 0.0)
    assert bool((err <= tol).all()), float((err - tol).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", [rov.ROPE_INTERLEAVED, rov.ROPE_HALVES])
@pytest.mark.parametrize("B,S,H,Hkv,d,rot,kw", [
    (1, 1, 1, 1, 2, 2, {}),                       # the smallest head
    (2, 5, 4, 2, 64, 64, {}),
    (1, 33, 3, 1, 128, 64, LINEAR),               # a part of the head
    (3, 7, 2, 2, 96, 48, PARTS),
    (2, 3, 2, 1, 80, 20, PARTS),                  # split pairs off 16 bytes
    (1, 4, 2, 1, 33, 10, {}),                     # odd head
    (1, 9, 1, 0, 512, 512, {}),                   # no keys, the longest head
    (1, 8200, 2, 1, 64, 64, {}),                  # four tokens a workgroup, the last one short of them (8192 + 8)
    (3, 2735, 1, 1, 40, 24, LINEAR),
])
@pytest.mark.parametrize("backward", [False, True])
def test_matches_formula(dtype, layout, B, S, H, Hkv, d, rot, kw, backward):
    print("rope", dtype, layout, B, S, H, Hkv, d, rot, backward, flush=True)
    g = torch.Generator().manual_seed(S * 7 + d)
    c = dict(rot=rot, theta=500000.0, layout=layout, **kw)
    Q = torch.randn(B, S, H, d, generator=g).to(DT[dtype]).cuda()
    K = torch.randn(B, S, Hkv, d, generator=g).to(DT[dtype]).cuda() if Hkv else None
    pos = torch.randint(0, 200000, (B, S), generator=g).cuda() if S % 2 else None
    cfg = rov.make_rope_cfg(**c)
    got = rov.rope(cfg, Q, K, positions=pos, backward=backward)
    for x, o in zip((Q, K), got if Hkv else (got,)):
        close(o, *reference(x, pos, c, backward), dtype)
        assert torch.equal(o[..., rot:], x[..., rot:])          # the rest of the head passes as it is


def test_positions_far_and_negative():
    c = dict(rot=64, theta=10000.0, layout=rov.ROPE_HALVES)
    Q = torch.randn(1, 6, 2, 64, generator=torch.Generator().manual_seed(1)).cuda()
    pos = torch.tensor([[0, -1, 1, 2 ** 20, 2 ** 24 + 1, -70000]]).cuda()
    close(rov.rope(rov.make_rope_cfg(**c), Q, positions=pos), *reference(Q, pos, c), "f32")
    # one row of positions serves all sequences
    Q2 = torch.randn(3, 6, 2, 64, generator=torch.Generator().manual_seed(2)).cuda()
    for p in (pos, pos[0]):
        close(rov.rope(rov.make_rope_cfg(**c), Q2, positions=p), *reference(Q2, pos, c), "f32")


@pytest.mark.parametrize("layout", [rov.ROPE_INTERLEAVED, rov.ROPE_HALVES])
@pytest.mark.parametrize("rot", [128, 32])
def test_in_place_inside_the_fused_product(layout, rot):
    # queries and keys of [q | k | v] rows turned where they lie: the same bits as out of place, and nothing else moves
    B, S, H, Hkv, d = 2, 37, 4, 2, 128
    qkv = torch.randn(B, S, H + 2 * Hkv, d, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    before = qkv.clone()
    cfg = rov.make_rope_cfg(rot, 10000.0, layout=layout)
    want = rov.rope(cfg, before[:, :, :H], before[:, :, H:H + Hkv])
    Q, K = qkv[:, :, :H], qkv[:, :, H:H + Hkv]
    rov.rope(cfg, Q, K, Qo=Q, Ko=K)
    assert torch.equal(Q, want[0]) and torch.equal(K, want[1]) and torch.equal(qkv[:, :, H + Hkv:], before[:, :, H + Hkv:])


def test_strides_and_surroundings():
    # [B, H, S, d] tensors seen as [B, S, H, d], results inside wider rows off 16 bytes: the rows' rest stays as it was
    B, S, H, d = 2, 11, 3, 64
    x = torch.randn(B, H, S, d, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).cuda()
    wide = torch.full((B, S, H, d + 6), 7.0, dtype=torch.bfloat16, device="cuda")
    c = dict(rot=64, theta=10000.0, layout=rov.ROPE_HALVES)
    out = wide[..., 3:3 + d]
    rov.rope(rov.make_rope_cfg(**c), x.transpose(1, 2), Qo=out)
    close(out, *reference(x.transpose(1, 2), None, c), "bf16")
    assert bool((wide[..., :3] == 7.0).all()) and bool((wide[..., 3 + d:] == 7.0).all())


def test_the_blocks_own_form_is_the_same_rotation():
    # adjacent pairs over the whole head at plain frequencies: what rov_block_forward applies, to bf16's half step
    c = dict(rot=128, theta=500000.0, layout=rov.ROPE_INTERLEAVED)
    Q = torch.randn(1, 64, 2, 128, generator=torch.Generator().manual_seed(5)).cuda()
    from oracle import dense as OD
    want = torch.from_numpy(OD.rope(Q.double().cpu().numpy(), 500000.0)) if hasattr(OD, "rope") else reference(Q, None, c)[0]
    close(rov.rope(rov.make_rope_cfg(**c), Q), want, reference(Q, None, c)[1], "f32")


def test_backward_is_the_transpose():
    # <R x, u> = <x, R^T u> for random u: the gradient of a rotation (with magnitude) is its transpose; both sides in fp32
    c = rov.make_rope_cfg(40, 10000.0, layout=rov.ROPE_HALVES, **PARTS)
    g = torch.Generator().manual_seed(6)
    x, u = (torch.randn(2, 50, 3, 64, generator=g).cuda() for _ in range(2))
    a = (rov.rope(c, x).double() * u.double()).sum()
    b = (x.double() * rov.rope(c, u, backward=True).double()).sum()
    # each side sums x.numel() products whose factors are off by 2^-21 (|a| + |b|) at most
    assert abs(float(a - b)) <= 2 * 2.0 ** -21 * 1.25 * 2 * float((x.abs().double() * u.abs().double()).sum() + x.numel())


def test_stream_and_graph():
    cfg = rov.make_rope_cfg(64, 10000.0, layout=rov.ROPE_HALVES)
    Q = torch.randn(4, 3, 2, 64, generator=torch.Generator().manual_seed(7)).cuda()
    pos = torch.randint(0, 5000, (4, 3)).cuda()
    want = rov.rope(cfg, Q, positions=pos)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = rov.rope(cfg, Q, positions=pos, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    out = torch.empty_like(Q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rov.rope(cfg, Q, positions=pos, Qo=out)
    for i in range(3):      # replays read what the buffers hold then
        pos += 17
        Q.mul_(1.5)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, rov.rope(cfg, Q, positions=pos)), i


def test_refusals_in_the_binding():
    cfg = rov.make_rope_cfg(64, 10000.0)
    Q = torch.zeros(1, 2, 2, 64, device="cuda")
    with pytest.raises(ValueError):
        rov.rope(cfg, Q.cpu())
    with pytest.raises(TypeError):
        rov.rope(cfg, Q, Q.to(torch.bfloat16))
    with pytest.raises(TypeError):
        rov.rope(cfg, Q, positions=torch.zeros(1, 2, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        rov.rope(cfg, Q, positions=torch.zeros(2, 2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        rov.rope(cfg, Q.transpose(2, 3))
    with pytest.raises(ValueError):
        rov.rope(cfg, Q, Qo=torch.zeros(1, 2, 2, 32, device="cuda"))
    with pytest.raises(rov.RovError):
        rov.rope(rov.make_rope_cfg(66, 10000.0), Q)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", [rov.ROPE_INTERLEAVED, rov.ROPE_HALVES])
def test_any_stride_and_address(dtype, layout):
    # heads that start off 16 bytes, in place: the bits of dense heads, and what lies around them stays
    B, S, H, d = 2, 19, 3, 64
    Q = torch.randn(B, S, H, d, generator=torch.Generator().manual_seed(4)).to(DT[dtype]).cuda()
    cfg = rov.make_rope_cfg(32, 10000.0, layout=layout)
    want = rov.rope(cfg, Q)
    wide = torch.full((B, S, H, d + 5), 3.0, dtype=DT[dtype], device="cuda")
    at = wide[..., 1:1 + d]
    at.copy_(Q)
    rov.rope(cfg, at, Qo=at)
    assert torch.equal(at, want) and bool((wide[..., :1] == 3.0).all()) and bool((wide[..., 1 + d:] == 3.0).all())
