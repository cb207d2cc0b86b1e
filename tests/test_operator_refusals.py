"""Argument checks of the operators around the block: refused on the host, before anything is enqueued (no GPU needed).

Pointers are numbers that look aligned and are never followed: every call here returns before a launch.
"""
import ctypes

import pytest

from paper_2410_07531_amd import binding as rov

P = 4096     # "pointers"
INVALID, UNSUPPORTED, WORKSPACE = rov.ERR_INVALID, rov.ERR_UNSUPPORTED, rov.ERR_WORKSPACE


def _rope(cfg=None, Q=P, Qo=2 * P, K=3 * P, Ko=4 * P, B=1, S=4, H=2, Hkv=1, d=64, strides=None, dtype=rov.BF16, positions=None, **c):
    cfg = rov.make_rope_cfg(**{"rot": 64, "theta": 1e4, **c}) if cfg is None else cfg
    st = [S * H * d, H * d, d] * 2 + [S * Hkv * d, Hkv * d, d] * 2 if strides is None else strides
    return rov.load().rov_rope(ctypes.byref(cfg), Q, Qo, K, Ko, B, S, H, Hkv, d, (ctypes.c_int64 * 12)(*st), dtype, positions, 0, 0, None)


@pytest.mark.parametrize("kw,code", [
    (dict(Q=0), INVALID), (dict(Qo=0), INVALID), (dict(K=0), INVALID), (dict(B=0), INVALID), (dict(S=-1), INVALID), (dict(H=0), INVALID),
    (dict(Hkv=-1), INVALID), (dict(d=0), INVALID), (dict(rot=66), INVALID), (dict(rot=3), INVALID), (dict(rot=0), INVALID),
    (dict(theta=0.0), INVALID), (dict(theta=float("inf")), INVALID), (dict(layout=2), INVALID), (dict(scaling=3), INVALID),
    (dict(scaling=rov.ROPE_SCALE_LINEAR, factor=0.0), INVALID), (dict(scaling=rov.ROPE_SCALE_PARTS, factor=8.0), INVALID),   # no trained length
    (dict(scaling=rov.ROPE_SCALE_PARTS, factor=8.0, trained_len=8, turns_low=4.0, turns_high=4.0), INVALID),
    (dict(magnitude=float("nan")), INVALID), (dict(dtype=7), INVALID), (dict(dtype=rov.FP8_E4M3), UNSUPPORTED), (dict(d=520, rot=64), UNSUPPORTED),
    (dict(Q=P + 1), INVALID), (dict(positions=P + 4), INVALID), (dict(Qo=P, strides=[512, 128, 64, 512, 128, 32] + [256, 64, 64] * 2), INVALID),   # in place, other strides
    (dict(Ko=2 * P), INVALID), (dict(Ko=P), INVALID), (dict(Qo=3 * P), INVALID),   # results over each other, over the other's input
    (dict(S=1 << 30, H=1, Hkv=0, rot=256, d=256, strides=[1 << 39, 512, 256] * 4), UNSUPPORTED),   # more workgroups than a launch has
])
def test_rope_refuses(kw, code):
    assert _rope(**kw) == code


def _norm(x=P, h=2 * P, w_post=P, gate=P, w_pre=P, y=3 * P, yn=4 * P, rows=8, n=64, ld=(64, 64, 64, 64), per=4, dtype=rov.BF16, xs=1.0, hs=1.0, eps=1e-5, fp8=0.0):
    return rov.load().rov_norm_residual(x, h, w_post, gate, w_pre, y, yn, rows, n, (ctypes.c_int64 * 4)(*ld), per, dtype, xs, hs, eps, fp8, None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=0), INVALID), (dict(h=0), INVALID), (dict(y=0), INVALID), (dict(yn=0), INVALID), (dict(w_pre=0), INVALID), (dict(rows=0), INVALID),
    (dict(n=0), INVALID), (dict(per=3), INVALID), (dict(per=0), INVALID), (dict(eps=0.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(xs=float("inf")), INVALID), (dict(dtype=9), INVALID), (dict(dtype=rov.FP8_E4M3), UNSUPPORTED), (dict(n=40000, ld=(40000,) * 4), UNSUPPORTED),
    (dict(ld=(64, 63, 64, 64)), INVALID), (dict(fp8=-1.0), INVALID), (dict(fp8=1.0, dtype=rov.F32), UNSUPPORTED), (dict(x=P + 1), INVALID),
    (dict(yn=3 * P), INVALID), (dict(fp8=1.0, yn=P), INVALID), (dict(y=P, ld=(64, 64, 72, 64)), INVALID), (dict(yn=2 * P, ld=(64, 72, 64, 64)), INVALID),
    (dict(rows=1 << 27, n=512, ld=(512,) * 4), UNSUPPORTED),   # more workgroups than a launch has
])
def test_norm_residual_refuses(kw, code):
    assert _norm(**kw) == code


def _norm_bwd(y=P, h=2 * P, w_post=P, gate=P, w_pre=P, dy=3 * P, dn=4 * P, dx=5 * P, dh=6 * P, dw_post=P, dgate=P, dw_pre=P, rows=8, n=64, ld=(64,) * 6, per=4,
              dtype=rov.BF16, eps=1e-5, ws=P, ws_bytes=1 << 30):
    return rov.load().rov_norm_residual_bwd(y, h, w_post, gate, w_pre, dy, dn, dx, dh, dw_post, dgate, dw_pre, rows, n, (ctypes.c_int64 * 6)(*ld), per,
                                            dtype, 1.0, 1.0, eps, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(y=0), INVALID), (dict(h=0), INVALID), (dict(dn=0), INVALID), (dict(w_pre=0), INVALID), (dict(w_pre=0, dn=0), INVALID),   # dw_pre without w_pre
    (dict(w_pre=0, dn=0, dw_pre=0, dy=0), INVALID), (dict(w_post=0), INVALID), (dict(gate=0), INVALID),
    (dict(dx=0, dh=0, dw_post=0, dgate=0, dw_pre=0), INVALID), (dict(rows=0), INVALID), (dict(per=5), INVALID), (dict(eps=-1.0), INVALID),
    (dict(n=40000, ld=(40000,) * 6), UNSUPPORTED), (dict(ld=(64, 64, 64, 64, 64, 8)), INVALID), (dict(ws=0), INVALID), (dict(ws=P + 4), INVALID),
    (dict(ws_bytes=16), WORKSPACE), (dict(dw_post=P + 2), INVALID), (dict(dtype=rov.FP8_E4M3), UNSUPPORTED),
    (dict(dh=5 * P), INVALID), (dict(dx=3 * P, ld=(64, 64, 64, 64, 72, 64)), INVALID),
])
def test_norm_residual_bwd_refuses(kw, code):
    assert _norm_bwd(**kw) == code


def _xent(X=P, W=P, t=P, M=4, V=10, K=8, ldx=8, ldw=8, dtype=rov.BF16, scale=1.0, ignore=-100, loss=5 * P, lse=6 * P, piece=0, ws=P, ws_bytes=1 << 30):
    return rov.load().rov_linear_xent(X, W, t, M, V, K, ldx, ldw, dtype, scale, ignore, loss, lse, piece, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(X=0), INVALID), (dict(W=0), INVALID), (dict(t=0), INVALID), (dict(loss=0), INVALID), (dict(lse=0), INVALID), (dict(M=0), INVALID),
    (dict(V=0), INVALID), (dict(K=-1), INVALID), (dict(ldx=7), INVALID), (dict(ldw=7), INVALID), (dict(ignore=3), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(piece=-1), INVALID), (dict(dtype=5), INVALID), (dict(dtype=rov.FP8_E4M3), UNSUPPORTED),
    (dict(ws=0), INVALID), (dict(ws=P + 16), INVALID), (dict(ws_bytes=64), WORKSPACE), (dict(X=P + 1), INVALID), (dict(t=P + 4), INVALID),
    (dict(lse=5 * P), INVALID), (dict(M=1 << 24, dtype=rov.F32), UNSUPPORTED), (dict(M=1 << 26, V=1 << 20), UNSUPPORTED),
])
def test_linear_xent_refuses(kw, code):
    assert _xent(**kw) == code


def _xent_bwd(X=P, W=P, t=P, lse=P, dloss=P, dlse=P, M=4, V=10, K=8, ldx=8, ldw=8, dtype=rov.BF16, ignore=-100, dX=5 * P, dW=6 * P, lddx=8, lddw=8, piece=0,
              ws=P, ws_bytes=1 << 30):
    return rov.load().rov_linear_xent_bwd(X, W, t, lse, dloss, dlse, M, V, K, ldx, ldw, dtype, 1.0, ignore, dX, dW, lddx, lddw, piece, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(X=0), INVALID), (dict(lse=0), INVALID), (dict(dloss=0), INVALID), (dict(dX=0, dW=0), INVALID), (dict(lddx=7), INVALID), (dict(lddw=4), INVALID),
    (dict(ignore=9), INVALID), (dict(dX=P + 1), INVALID), (dict(ws=0), INVALID), (dict(ws_bytes=64), WORKSPACE), (dict(dtype=rov.FP8_E4M3), UNSUPPORTED),
    (dict(dlse=P + 2), INVALID), (dict(K=0), INVALID), (dict(dW=5 * P), INVALID),
])
def test_linear_xent_bwd_refuses(kw, code):
    assert _xent_bwd(**kw) == code


def test_workspace_sizes():
    assert rov.norm_residual_bwd_workspace_bytes(8, 64, 3, rov.BF16) == 0 and rov.norm_residual_bwd_workspace_bytes(8, 64, 8, rov.FP8_E4M3) == 0
    assert rov.norm_residual_bwd_workspace_bytes(8, 64, 8, rov.BF16) > 0
    assert rov.linear_xent_workspace_bytes(0, 10, 8, rov.BF16) == 0 and rov.linear_xent_workspace_bytes(4, 10, 8, rov.FP8_E4M3) == 0
    whole, small = (rov.linear_xent_workspace_bytes(512, 60000, 256, rov.BF16, backward=True, vocab_piece=p) for p in (60000, 1024))
    assert 0 < small < whole
    # no piece keeps the logits of a long batch
    assert rov.linear_xent_workspace_bytes(65536, 131072, 4096, rov.BF16) < 65536 * 131072 * 4 // 4
