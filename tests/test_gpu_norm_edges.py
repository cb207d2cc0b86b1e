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
