"""Blocks with their own rotary form, post norms, gates and residual scales under the schedules that run ahead: hybrid, and masks left in
flight between blocks.  Every schedule drops the same elements, so outputs are those of the sequential one, bit for bit.
"""
import pytest
import torch

import test_gpu_operators_together as T
from paper_2410_07531_amd import binding as rov
from paper_2410_07531_amd import workloads as wl

pytestmark = pytest.mark.gpu
B, S, P, OFFSET = 2, 160, 0.1, 640
DIMS = {**T.DIMS, "ffn": 1024}


def _block(causal, fp8):
    x, w, around, pos = T._setup(B, S, 81)
    names = ("wqkv", "wo", "wg", "wu", "wd")
    w = {k: (v[:1024].contiguous() if k in ("wg", "wu") else v[:, :1024].contiguous() if k == "wd" else v) for k, v in w.items()}
    dims = tuple(DIMS[k] for k in ("H", "Hkv", "d", "hidden", "ffn"))
    if fp8:
        scale = {n: float(w[n].abs().max()) / 448.0 for n in names}
        w = {n: ((w[n].float() / scale[n]).to(torch.float8_e4m3fn).view(torch.uint8) if n in names else w[n]) for n in w}
        weights = rov.make_block_weights(w, scale)
        cfg = rov.make_block_cfg(*dims, P, causal=causal, dtype=rov.FP8_E4M3, act_scale=[5.0 / 448, 4.0 / 448, 5.0 / 448, 2.0 / 448])
    else:
        weights, cfg = rov.make_block_weights(w), rov.make_block_cfg(*dims, P, causal=causal)
    form = rov.make_rope_cfg(**T.ROPE)
    opts = rov.make_block_opts(rope=form, positions=pos, rows_per_gate=S, x_scale=0.9, h_scale=0.5, **around)
    ws = torch.empty(rov.block_workspace_bytes(cfg, B, S, 0), dtype=torch.uint8, device="cuda")
    main, side = torch.cuda.Stream(), torch.cuda.Stream()
    calls = rov.mask_philox_calls(B, DIMS["H"], S)

    def run(y, sched, layer, mask, **kw):
        rov.block_forward(weights, x, y, cfg, sched, wl.SEED, OFFSET + layer * calls, mask, ws, main, side, opts=kw.pop("opts", opts), **kw)

    run.keep = (x, w, around, pos, form)
    return x, run, cfg


def _masks(n):
    return [torch.full(rov.mask_shape(B, DIMS["H"], S), 0x2AAAAAAAAAAAAAAA, dtype=torch.int64, device="cuda") for _ in range(n)]


def _sequential(x, run, layers):
    m, ys = _masks(1)[0], [torch.zeros_like(x) for _ in range(layers)]
    torch.cuda.synchronize()
    for layer, y in enumerate(ys):
        run(y, rov.SCHED_SEQUENTIAL, layer, m)
    torch.cuda.synchronize()
    plain = torch.zeros_like(x)
    torch.cuda.synchronize()
    run(plain, rov.SCHED_SEQUENTIAL, 0, m, opts=None)
    torch.cuda.synchronize()
    assert not torch.equal(ys[0], ys[1]) and not torch.equal(ys[0], plain) and bool(torch.isfinite(ys[0]).all())
    return ys


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("rows", [-1, 64, 100, 160])
def test_hybrid(rows, causal, fp8):
    # no row, some, all of them with stored bits; the block's own mask, then one that the block before made
    print("block options, hybrid", rows, causal, fp8, flush=True)
    x, run, cfg = _block(causal, fp8)
    want = _sequential(x, run, 2)
    prev = rov.set_block_hybrid_mask_rows(rows)
    try:
        assert rov.block_hybrid_mask_rows(cfg, B, S) == max(0, rows - rows % 32)
        m0, m1 = _masks(2)
        ys = [torch.zeros_like(x) for _ in range(2)]
        torch.cuda.synchronize()
        run(ys[0], rov.SCHED_HYBRID, 0, m0, next_mask=m1)
        run(ys[1], rov.SCHED_HYBRID, 1, m1, mask_ready=rov.MASK_READY, next_mask=m0)
        torch.cuda.synchronize()
    finally:
        rov.set_block_hybrid_mask_rows(prev)
    assert torch.equal(ys[0], want[0]) and torch.equal(ys[1], want[1])


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("tiny_grid", [False, True])
def test_masks_in_flight_over_three_blocks(tiny_grid, causal, fp8):
    # layer 0 makes its own mask, layers 1 and 2 find theirs in flight; options that are refused leave the mask in flight
    print("block options, deferred", tiny_grid, causal, fp8, flush=True)
    x, run, cfg = _block(causal, fp8)
    want = _sequential(x, run, 3)
    bad = rov.make_block_opts(x_scale=float("nan"))
    prev = rov.set_rng_max_workgroups(1) if tiny_grid else None
    try:
        masks, ys = _masks(2), [torch.zeros_like(x) for _ in range(3)]
        torch.cuda.synchronize()
        run(ys[0], rov.SCHED_OVERLAP_DEFERRED, 0, masks[0], next_mask=masks[1])
        with pytest.raises(rov.RovError) as e:
            run(ys[1], rov.SCHED_OVERLAP_DEFERRED, 1, masks[1], mask_ready=rov.MASK_IN_FLIGHT, next_mask=masks[0], opts=bad)
        assert e.value.code == rov.ERR_INVALID
        run(ys[1], rov.SCHED_OVERLAP_DEFERRED, 1, masks[1], mask_ready=rov.MASK_IN_FLIGHT, next_mask=masks[0])
        run(ys[2], rov.SCHED_OVERLAP, 2, masks[0], mask_ready=rov.MASK_IN_FLIGHT)
        torch.cuda.synchronize()
    finally:
        if tiny_grid:
            rov.set_rng_max_workgroups(prev)
    assert all(torch.equal(y, w) for y, w in zip(ys, want))
