"""What the operators around the block refuse on the host, in the binding and in the library, and what their workspaces go by (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2410_07531_amd import binding as rov


@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-50, -1.0, float("nan")])
@pytest.mark.parametrize("given", [False, True])
def test_a_scale_of_zero_does_not_ask_for_two_bytes_an_element(scale, given):
    # the library takes a scale of 0 as "yn in x's type": bf16 values in a buffer of bytes would end behind it
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.ones(64, dtype=torch.bfloat16)
    yn = torch.zeros(4, 64, dtype=torch.uint8) if given else None
    with pytest.raises(ValueError, match="yn_fp8_scale"):
        rov.norm_residual(x, x, w_pre=w, yn=yn, yn_fp8_scale=scale)


class _NotAsked:
    def __getattr__(self, name):
        raise AssertionError("%s was asked with sizes that a C int does not hold" % name)


BIG = 2 ** 32 + 8      # a C int would hold 8


def _calls_with_big_sizes():
    t = lambda *shape, dtype=torch.bfloat16: torch.empty(*shape, dtype=dtype, device="meta")   # (no memory behind them)
    cfg = rov.make_rope_cfg(8, 1e4)
    for at in range(4):
        shape = [1, 2, 2, 8]
        shape[at] = BIG
        yield "rope %d" % at, lambda shape=shape: rov.rope(cfg, t(*shape))
    yield "rope keys", lambda: rov.rope(cfg, t(1, 2, 2, 8), t(1, 2, BIG, 8))
    yield "rope form", lambda: rov.make_rope_cfg(BIG, 1e4)
    yield "rope form, trained length", lambda: rov.make_rope_cfg(8, 1e4, trained_len=BIG)
    yield "norm", lambda: rov.norm_residual(t(1, BIG), t(1, BIG))
    yield "norm back", lambda: rov.norm_residual_bwd(None, None, t(1, BIG))
    for M, V, K, piece in ((BIG, 4, 8, 0), (4, BIG, 8, 0), (4, 4, BIG, 0), (4, 4, 8, BIG)):
        args = (t(M, K), t(V, K), t(M, dtype=torch.int64))
        f = t(M, dtype=torch.float32)
        yield "loss %d %d %d %d" % (M, V, K, piece), lambda args=args, piece=piece: rov.linear_xent(*args, vocab_piece=piece)
        yield "loss back %d %d %d %d" % (M, V, K, piece), lambda args=args, f=f, piece=piece: rov.linear_xent_bwd(*args, f, f, vocab_piece=piece)


@pytest.mark.parametrize("name,call", list(_calls_with_big_sizes()), ids=lambda v: v.replace(" ", "_") if isinstance(v, str) else "")
def test_sizes_that_a_c_int_does_not_hold(monkeypatch, name, call):
    monkeypatch.setattr(rov, "_on_gpu", lambda *a: None)
    monkeypatch.setattr(rov, "_torch", torch)
    monkeypatch.setattr(rov, "load", lambda: _NotAsked())
    monkeypatch.setattr(rov, "_stream_ptr", lambda stream: 0)
    with pytest.raises(rov.RovError) as e:
        call()
    assert e.value.code == rov.ERR_UNSUPPORTED


def test_workspaces_of_sizes_that_a_c_int_does_not_hold():
    for sizes in ((BIG, 10, 8), (4, BIG, 8), (4, 10, BIG)):
        assert rov.linear_xent_workspace_bytes(*sizes, rov.BF16) == 0
    assert rov.linear_xent_workspace_bytes(4, 10, 8, rov.BF16, True, BIG) == 0
    assert rov.norm_residual_bwd_workspace_bytes(8, BIG, 8, rov.BF16) == 0


@pytest.mark.parametrize("dtype", [rov.BF16, rov.F32])
def test_gradients_over_the_other_operand_are_refused_by_the_library(dtype):
    # pointers that are never followed: one piece's gradients over an operand that the next piece reads
    X, W, dX, dW = 4096, 8192, 12288, 16384
    call = lambda dX, dW: rov.load().rov_linear_xent_bwd(X, W, 4096, 4096, 4096, None, 8, 8, 8, 8, 8, dtype, 1.0, -100, dX, dW, 8, 8, 0, 4096, 0, None)
    assert call(dX, dW) == rov.ERR_WORKSPACE        # (nothing else is wrong with the call)
    assert call(W, dW) == call(dX, X) == call(W, X) == call(W, None) == call(None, X) == rov.ERR_INVALID


def test_a_block_whose_norms_have_too_many_rows_is_refused_before_anything_runs():
    # 4.2 million tokens of 4160 values are more workgroups than a launch of the norm behind the branch has; pointers are never followed
    P, hidden = 1 << 20, 4160
    cfg = rov.make_block_cfg(1, 1, 64, hidden, 64, 0.0)
    w = rov.BlockWeights(*[P] * 7, (ctypes.c_float * 5)(*[1.0] * 5))
    opts = rov.BlockOpts(None, None, 0, P, None, None, None, 0, 1.0, 1.0)
    call = lambda B: rov.load().rov_block_forward_opts(ctypes.byref(w), ctypes.byref(opts), P, 2 * P, B, 129, ctypes.byref(cfg), rov.SCHED_FUSED, 1, 0, 0, None, None,
                                                       P, 1 << 62, None, None)
    assert call(1 << 15) == rov.ERR_UNSUPPORTED


def test_what_the_piece_of_the_vocabulary_sets():
    # the bf16 loss keeps no logits: its workspace does not depend on the piece; fp32's does, and both gradients'
    size = lambda dtype, backward, piece: rov.linear_xent_workspace_bytes(512, 60000, 256, dtype, backward, piece)
    assert size(rov.BF16, False, 0) == size(rov.BF16, False, 1024) == size(rov.BF16, False, 60000) > 0
    for dtype, backward in ((rov.F32, False), (rov.F32, True), (rov.BF16, True)):
        assert 0 < size(dtype, backward, 1024) < size(dtype, backward, 60000)
