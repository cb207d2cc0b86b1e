"""Gradients of the norms around a block at the ends of their range: as many gates as a call may have, branches that hold
infinities, rows far from one, rows of zeros.
"""
import pytest
import torch

from paper_2410_07531_amd import binding as rov

pytestmark = pytest.mark.gpu


def test_as_many_gates_as_a_call_may_have():
    # one gate a row, 2^31 - 1 rows of one element: a workgroup's step to its next gate leaves 32 bits behind the last one.  Results
    # are one rounded product each, compared bit for bit.
    rows = 2 ** 31 - 1
    print("norm bwd", rows, "gates", flush=True)
    part = torch.randn(2 ** 20 + 7, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    dy, h, gate = (part.roll(k).repeat(rows // part.numel() + 1)[:rows].view(rows, 1) for k in (0, 1, 2))
    dx, dh, _, _, dgate = rov.norm_residual_bwd(None, h, dy, gate=gate)
    for at in range(0, rows, 2 ** 28):
        a, b, g = (v[at:at + 2 ** 28].float() for v in (dy, h, gate))
        assert torch.equal(dx[at:at + 2 ** 28], dy[at:at + 2 ** 28]), at
        assert torch.equal(dh[at:at + 2 ** 28], (a * g).to(torch.bfloat16)) and torch.equal(dgate[at:at + 2 ** 28], a * b), at
    del dy, h, gate, dx, dh, dgate, a, b, g
    torch.cuda.empty_cache()


# Tolerances below: as in the tests of the gradients at ordinary sizes, 2^-17 of the terms' magnitudes and, for bf16, half a step, 2^-8, of the value.
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def near(got, want, mag, dtype, rel=2.0 ** -17):
    got, want, mag = got.double().cpu(), want.cpu(), mag.cpu()
    assert torch.equal(torch.isfinite(got), torch.isfinite(want))
    err = (got - want).abs()
    fine = torch.isfinite(want)
    tol = rel * mag + (2.0 ** -8 * want.abs() if dtype == "bf16" else 0.0)
    assert bool((err <= tol)[fine].all()), float((err - tol)[fine].max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [100, 512, 1030, 9000])      # element by element, whole pieces, ragged pieces, rows that are read twice
@pytest.mark.parametrize("gated,pre", [(True, False), (True, True), (False, False), (False, True)])
def test_without_a_norm_behind_the_branch_its_gradient_does_not_depend_on_it(dtype, n, gated, pre):
    # dh = h_scale * gate * gy: infinities and NaN in h reach dgate, where they belong, and not dh
    rows = 6
    g = torch.Generator().manual_seed(n)
    r = lambda *s: torch.randn(*s, generator=g).to(DT[dtype]).cuda()
    h, dy, y, dn, gate, w = r(rows, n), r(rows, n), r(rows, n), r(rows, n), r(2, n), 1 + 0.1 * r(n)
    h[0, 3], h[1, n - 1], h[2, 7], h[5] = float("inf"), -float("inf"), float("nan"), float("inf")
    kw = dict(w_pre=w) if pre else {}
    dx, dh, dw_pre, _, dgate = rov.norm_residual_bwd(y if pre else None, h, dy, dn if pre else None, gate=gate if gated else None, h_scale=0.5, **kw)
    gy, mag = dy.double(), dy.double().abs()
    if pre:
        Y, t = y.double(), dn.double() * w.double()
        q = 1.0 / torch.sqrt((Y * Y).mean(1, keepdim=True) + 1e-5)
        gy = gy + q * t - Y * q ** 3 * (Y * t).mean(1, keepdim=True)
        mag = mag + q * t.abs() + Y.abs() * q ** 3 * (Y * t).abs().mean(1, keepdim=True)
        near(dw_pre, (dn.double() * Y * q).sum(0), (dn.double() * Y * q).abs().sum(0), "f32", 2.0 ** -16)
    spread = gate.double().repeat_interleave(3, 0) if gated else 1.0
    near(dx, gy, mag, dtype)
    near(dh, 0.5 * spread * gy, 0.5 * mag * (spread.abs() if gated else 1.0), dtype)
    if gated:
        near(dgate, (0.5 * gy * h.double()).view(2, 3, n).sum(1), (0.5 * mag * h.double().abs()).view(2, 3, n).sum(1), "f32", 2.0 ** -16)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [72, 100, 1030, 9000])
@pytest.mark.parametrize("size,eps", [(1e13, 1e-5), (1e15, 1e-5), (1e17, 1e-5), (1e-13, 1e-28), (1e-15, 1e-32), (0.0, 1e-30)])
def test_rows_far_from_one_and_rows_of_zeros(dtype, n, size, eps):
    # dx and dh are of the size of dn / size (dn is sent in that large, so that they are of the size of one) and each is a difference of two
    # terms as large as it: hat's and h_hat's means must not vanish, nor 0 times a factor beyond fp32 become NaN.  Branch and stream lean on their
    # gradients, so that the means are 0.3 to 0.7 and not near 0.
    rows, f64 = 4, torch.float64
    g = torch.Generator().manual_seed(n + 1)
    r = lambda *s: torch.randn(*s, generator=g)
    to = lambda v: v.to(DT[dtype]).cuda()
    dn, q0 = r(rows, n), r(rows, n)
    gain = size if size else 1.0
    y, h = to(size * (0.5 * dn + r(rows, n))), to(size * (0.5 * q0 + r(rows, n)))
    w_pre, w_post, gate = to(1 + 0.1 * r(n)), to(1 + 0.1 * r(n)), to(0.5 + 0.1 * r(n))
    dn, dy = to(gain * dn), to(q0)
    dx, dh, dw_pre, dw_post, dgate = rov.norm_residual_bwd(y, h, dy, dn, w_pre, w_post, gate, h_scale=0.5, eps=eps)
    Y, H, DN, DY, WN, WP, GT = (v.to(f64) for v in (y, h, dn, dy, w_pre, w_post, gate))
    mean = lambda v: v.mean(1, keepdim=True)
    ry, rh = 1 / torch.sqrt(mean(Y * Y) + eps), 1 / torch.sqrt(mean(H * H) + eps)
    hat, hh, t = Y * ry, H * rh, WN * DN
    if size:
        assert float((mean(hat * t) / gain).abs().min()) > 0.1
    gy, my = DY + ry * (t - hat * mean(hat * t)), DY.abs() + ry * (t.abs() + hat.abs() * mean((hat * t).abs()))
    q, mq = 0.5 * GT * gy * WP, 0.5 * (GT * WP).abs() * my
    near(dx, gy, my, dtype)
    near(dh, rh * (q - hh * mean(hh * q)), rh * (mq + hh.abs() * mean(hh.abs() * mq)), dtype)
    near(dw_pre, (DN * hat).sum(0), (DN * hat).abs().sum(0), "f32", 2.0 ** -16)
    near(dw_post, (0.5 * GT * gy * hh).sum(0), (0.5 * GT.abs() * my * hh.abs()).sum(0), "f32", 2.0 ** -16)
    near(dgate, (0.5 * WP * gy * hh).sum(0), (0.5 * WP.abs() * my * hh.abs()).sum(0), "f32", 2.0 ** -16)
