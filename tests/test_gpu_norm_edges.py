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
