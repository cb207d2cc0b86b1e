"""Loss over the vocabulary and its gradients against the definition in 64 bits.

Tolerances.  A logit is a sum of K products in fp32: off by at most K * 2^-24 of scale * sum |x w| (dz below, the largest
of the row).  exp and log add 2^-21 of a sum of positives and 2^-23 of their result, so lse and loss are off by at most
2 dz + 2^-20 + 2^-22 |lse|.  A gradient logit G is off by (2 dz + 2^-19) of its two terms' magnitudes, and, for bf16, by a half step, 2^-8, of itself;
for dW the rows of X, times their factors, are rounded too: another 2^-8 of each term;
products over V (dX) and M (dW) terms carry that and add V (M) * 2^-24 of the sum of magnitudes; bf16 results another 2^-8.
Below the smallest normal number, 2^-126, fp32 has no relative precision (exp and the matrix products flush there): a term
of G (|dloss + dlse| < 4) is off by up to 4 * 2^-126, its product with w or x by another 2^-126, V (M) of them in a sum.
"""
import pytest
import torch

from paper_2410_07531_amd import binding as rov

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(M, V, K, dtype, seed=0, ignored=0.2, sd=1.0):
    g = torch.Generator().manual_seed(seed + 1000 * M + V + K)
    W = (torch.randn(V, K, generator=g) * 2.0 / K ** 0.5).to(DT[dtype])
    t = torch.randint(0, V, (M,), generator=g)
    X = (sd * torch.randn(M, K, generator=g) + W[t].float() * K / 4).to(DT[dtype])
    t[torch.rand(M, generator=g) < ignored] = -100
    dloss, dlse = torch.rand(M, generator=g) + 0.5, 0.3 * torch.randn(M, generator=g)
    return [v.cuda() for v in (X, W, t, dloss, dlse)]


def reference(X, W, t, dloss=None, dlse=None, scale=1.0, ignore=-100):
    """Results and tolerances in float64 (on the GPU in float64, elementary operations)."""
    bf16 = X.dtype == torch.bfloat16
    X, W = X.double(), W.double()
    M, K = X.shape
    V = W.shape[0]
    z = scale * (X @ W.t())
    dz = K * 2.0 ** -24 * abs(scale) * (X.abs() @ W.abs().t()).amax(1)
    lse = torch.logsumexp(z, 1)
    keep = t != ignore
    at = torch.where(keep, t, torch.zeros_like(t))[:, None]
    loss = torch.where(keep, lse - z.gather(1, at)[:, 0], torch.zeros_like(lse))
    out = dict(loss=loss, lse=lse, tol=2 * dz + 2.0 ** -20 + 2.0 ** -22 * lse.abs())
    if dloss is None:
        return out
    a = dloss.double() * keep
    b = a + (0.0 if dlse is None else dlse.double() * keep)
    G = torch.exp(z - lse[:, None]) * b[:, None]
    mag = G.abs().scatter_add(1, at, a.abs()[:, None])
    G = scale * G.scatter_add(1, at, -a[:, None])
    err = abs(scale) * mag * (2 * dz + 2.0 ** -19)[:, None] + (2.0 ** -8 * G.abs() if bf16 else 0.0)
    mag = mag * abs(scale)
    Xk = X * keep[:, None]
    out["dX"], out["dW"] = G @ W, G.t() @ Xk
    half = 2.0 ** -8 if bf16 else 2.0 ** -24
    out["tX"] = err @ W.abs() + V * 2.0 ** -24 * (mag @ W.abs()) + half * out["dX"].abs()
    errW = err + (2.0 ** -8 * G.abs() if bf16 else 0.0)
    out["tW"] = errW.t() @ Xk.abs() + M * 2.0 ** -24 * (mag.t() @ Xk.abs()) + half * out["dW"].abs()
    out["tX"] += V * 2.0 ** -126 * (1 + 4 * W.abs().max())
    out["tW"] += M * 2.0 ** -126 * (1 + 4 * Xk.abs().max())
    return out


def close(got, want, tol, what):
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), (what, float((err - tol).max()), float(err.max()))


SIZES = [(1, 1, 1, 0), (1, 300, 8, 0), (3, 5, 7, 0), (17, 1000, 64, 0), (64, 257, 128, 0), (130, 2050, 96, 512), (257, 999, 130, 256), (300, 1300, 264, 0),
         (33, 5003, 513, 1024), (512, 4096, 512, 0), (513, 2049, 1000, 700), (1025, 777, 72, 0), (2, 70001, 40, 0),
         # more than a round of 256 x 256 tiles and a rest in narrower ones: columns, columns of packed operands, rows of dX
         (300, 70001, 64, 0), (300, 40001, 33, 0), (66000, 300, 16, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,V,K,piece", SIZES)
def test_loss(dtype, M, V, K, piece):
    print("xent", dtype, M, V, K, piece, flush=True)
    X, W, t, _, _ = make(M, V, K, dtype)
    r = reference(X, W, t, scale=0.7)
    loss, lse = rov.linear_xent(X, W, t, scale=0.7, vocab_piece=piece)
    close(lse, r["lse"], r["tol"], "lse")
    close(loss, r["loss"], r["tol"], "loss")
    assert bool((loss[t == -100] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,V,K,piece", SIZES)
@pytest.mark.parametrize("with_dlse", [False, True])
def test_gradients(dtype, M, V, K, piece, with_dlse):
    print("xent bwd", dtype, M, V, K, piece, with_dlse, flush=True)
    X, W, t, dloss, dlse = make(M, V, K, dtype, seed=1)
    dlse = dlse if with_dlse else None
    r = reference(X, W, t, dloss, dlse, scale=0.7)
    _, lse = rov.linear_xent(X, W, t, scale=0.7, vocab_piece=piece)
    dX, dW = rov.linear_xent_bwd(X, W, t, lse, dloss, dlse, scale=0.7, vocab_piece=piece)
    assert dX.dtype == X.dtype and dW.dtype == X.dtype
    close(dX, r["dX"], r["tX"], "dX")
    close(dW, r["dW"], r["tW"], "dW")
    again = rov.linear_xent_bwd(X, W, t, lse, dloss, dlse, scale=0.7, vocab_piece=piece)
    assert torch.equal(dX, again[0]) and torch.equal(dW, again[1])
    one = rov.linear_xent_bwd(X, W, t, lse, dloss, dlse, scale=0.7, vocab_piece=piece, need_dW=False)
    other = rov.linear_xent_bwd(X, W, t, lse, dloss, dlse, scale=0.7, vocab_piece=piece, need_dX=False)
    assert one[1] is None and other[0] is None and torch.equal(one[0], dX) and torch.equal(other[1], dW)


def test_pieces_by_the_librarys_rule():
    # enough rows that the library cuts the vocabulary itself
    M, V, K = 4096, 33000, 64
    X, W, t, dloss, _ = make(M, V, K, "bf16", seed=2)
    size = lambda piece: rov.linear_xent_workspace_bytes(M, V, K, rov.BF16, True, piece)
    assert size(0) == size(32768) != size(V)
    r = reference(X, W, t, dloss)
    loss, lse = rov.linear_xent(X, W, t)
    close(loss, r["loss"], r["tol"], "loss")
    dX, dW = rov.linear_xent_bwd(X, W, t, lse, dloss)
    close(dX, r["dX"], r["tX"], "dX")
    close(dW, r["dW"], r["tW"], "dW")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_operands_and_surroundings(dtype):
    M, V, K = 70, 900, 128
    X, W, t, dloss, _ = make(M, V, K, dtype, seed=3)
    for pad in (8, 3):       # rows on and off 16 bytes
        Xw, Ww = (torch.full((v.shape[0], K + 2 * pad), float("nan"), dtype=v.dtype, device="cuda") for v in (X, W))
        Xs, Ws = Xw[:, pad:pad + K], Ww[:, pad:pad + K]
        Xs.copy_(X)
        Ws.copy_(W)
        dXw, dWw = (torch.full_like(v, 5.0) for v in (Xw, Ww))
        r = reference(X, W, t, dloss)
        loss, lse = rov.linear_xent(Xs, Ws, t, vocab_piece=512)
        close(loss, r["loss"], r["tol"], "loss")
        dX, dW = rov.linear_xent_bwd(Xs, Ws, t, lse, dloss, dX=dXw[:, pad:pad + K], dW=dWw[:, pad:pad + K], vocab_piece=512)
        close(dX, r["dX"], r["tX"], "dX")
        close(dW, r["dW"], r["tW"], "dW")
        for w in (dXw, dWw):
            assert bool((w[:, :pad] == 5.0).all()) and bool((w[:, pad + K:] == 5.0).all())


def test_rows_of_w_that_reach_beyond_4_gib():
    # 640 rows, 8 MiB apart: the gradients' products take packed pieces instead
    M, V, K = 40, 600, 64
    X, W, t, dloss, _ = make(M, V, K, "bf16", seed=10)
    far = torch.empty(V * 2 ** 22, dtype=torch.bfloat16, device="cuda").view(V, 2 ** 22)[:, 8:8 + K]
    far.copy_(W)
    r = reference(X, W, t, dloss)
    loss, lse = rov.linear_xent(X, far, t)
    close(loss, r["loss"], r["tol"], "loss")
    dX, dW = rov.linear_xent_bwd(X, far, t, lse, dloss)
    close(dX, r["dX"], r["tX"], "dX")
    close(dW, r["dW"], r["tW"], "dW")
    with pytest.raises(rov.RovError) as e:      # 256 rows of X beyond 4 GiB
        rov.linear_xent(torch.empty(2 ** 24 + 64, dtype=torch.bfloat16, device="cuda").as_strided((2, K), (2 ** 24, 1)), W, t[:2])
    assert e.value.code == rov.ERR_UNSUPPORTED


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ignored_rows_may_hold_anything(dtype):
    # padding: NaN and infinity in the hidden states and in the gradients of ignored rows reach nothing
    M, V, K = 100, 600, 64
    X, W, t, dloss, dlse = make(M, V, K, dtype, seed=4)
    t[::3] = -100
    r = reference(X, W, t, dloss, dlse)
    bad = t == -100
    X[bad] = float("nan")
    X[3] = float("inf")
    dloss[bad], dlse[bad] = float("nan"), float("inf")
    loss, lse = rov.linear_xent(X, W, t)
    close(loss, r["loss"], r["tol"] + bad * 0.0, "loss")
    dX, dW = rov.linear_xent_bwd(X, W, t, lse, dloss, dlse)
    close(dX, r["dX"], r["tX"], "dX")
    close(dW, r["dW"], r["tW"], "dW")
    assert bool((dX[bad] == 0).all())


def test_all_rows_ignored():
    X, W, t, dloss, _ = make(20, 300, 64, "bf16", seed=5)
    t[:] = 777
    loss, lse = rov.linear_xent(X, W, t, ignore_index=777)
    dX, dW = rov.linear_xent_bwd(X, W, t, lse, dloss, ignore_index=777)
    assert bool((loss == 0).all()) and bool((dX == 0).all()) and bool((dW == 0).all()) and bool(torch.isfinite(lse).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_targets_outside_the_vocabulary_show(dtype):
    X, W, t, dloss, _ = make(40, 300, 64, dtype, seed=6, ignored=0.0)
    good = reference(X, W, t)
    t[5], t[9], t[11] = 300, -1, 2 ** 40
    loss, lse = rov.linear_xent(X, W, t)
    out = torch.zeros(40, dtype=torch.bool, device="cuda")
    out[[5, 9, 11]] = True
    assert bool(torch.isnan(loss[out]).all())
    close(lse, good["lse"], good["tol"], "lse")
    close(loss[~out], good["loss"][~out], good["tol"][~out], "loss")
    dX, dW = rov.linear_xent_bwd(X, W, t, lse, dloss)
    assert bool(torch.isnan(dX[out]).all()) and bool(torch.isfinite(dX[~out]).all()) and bool(torch.isnan(dW).any())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_logits_far_apart(dtype):
    # logits of hundreds, some of them equal, one row flat: maxima are taken out before exp
    M, V, K = 8, 1030, 64
    X, W, t, dloss, _ = make(M, V, K, dtype, seed=7, ignored=0.0)
    X = X * 64
    X[2] = 0
    W[17] = W[900]
    r = reference(X, W, t, dloss)
    loss, lse = rov.linear_xent(X, W, t, vocab_piece=256)
    close(lse, r["lse"], r["tol"], "lse")
    close(loss, r["loss"], r["tol"], "loss")
    dX, dW = rov.linear_xent_bwd(X, W, t, lse, dloss, vocab_piece=256)
    close(dX, r["dX"], r["tX"], "dX")
    close(dW, r["dW"], r["tW"], "dW")


def test_gradient_against_differences():
    X, W, t, dloss, dlse = make(12, 80, 24, "f32", seed=8)
    X = X * 0.3
    f = lambda X, W: float((lambda r: (r[0].double() * dloss.double()).sum() + (r[1].double() * dlse.double() * (t != -100)).sum())(rov.linear_xent(X, W, t)))
    lse = rov.linear_xent(X, W, t)[1]
    dX, dW = rov.linear_xent_bwd(X, W, t, lse, dloss, dlse)
    g = torch.Generator().manual_seed(8)
    for which, grad in (("X", dX), ("W", dW)):
        u = torch.randn(grad.shape, generator=g).cuda()
        step = 4e-3
        plus, minus = (f(X + s * u, W) if which == "X" else f(X, W + s * u) for s in (step, -step))
        slope = float((grad.double() * u.double()).sum())
        # 12 losses of size up to 10, each off by 2^-20 of that, over the step; third-order term of the softmax
        assert abs((plus - minus) / (2 * step) - slope) <= 12 * 10 * 2.0 ** -20 / step + 1e-2 * (1 + abs(slope)), which


def test_stream_and_graph():
    X, W, t, dloss, _ = make(200, 1500, 128, "bf16", seed=9)
    loss, lse = rov.linear_xent(X, W, t, vocab_piece=512)
    want = rov.linear_xent_bwd(X, W, t, lse, dloss, vocab_piece=512)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    l2, s2 = rov.linear_xent(X, W, t, vocab_piece=512, stream=side)
    got = rov.linear_xent_bwd(X, W, t, s2, dloss, vocab_piece=512, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(l2, loss) and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a = rov.linear_xent(X, W, t, vocab_piece=512)
        b = rov.linear_xent_bwd(X, W, t, a[1], dloss, vocab_piece=512)
    for i in range(3):
        X.mul_(0.9)
        t.copy_(t.roll(1))
        graph.replay()
        torch.cuda.synchronize()
        c = rov.linear_xent(X, W, t, vocab_piece=512)
        d = rov.linear_xent_bwd(X, W, t, c[1], dloss, vocab_piece=512)
        assert all(torch.equal(x, y) for x, y in zip(a + b, c + d)), i


def test_refusals_in_the_binding():
    X, W, t = torch.zeros(4, 16, device="cuda"), torch.zeros(30, 16, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    f = torch.zeros(4, device="cuda")
    for bad in ((X, W[:, :8], t), (X, W, t[:3]), (X.cpu(), W, t), (X.t().contiguous().t(), W, t)):
        with pytest.raises(ValueError):
            rov.linear_xent(*bad)
    with pytest.raises(TypeError):
        rov.linear_xent(X, W.to(torch.bfloat16), t)
    with pytest.raises(TypeError):
        rov.linear_xent(X, W, t.to(torch.int32))
    with pytest.raises(TypeError):
        rov.linear_xent_bwd(X, W, t, f.double(), f)
    with pytest.raises(ValueError):
        rov.linear_xent_bwd(X, W, t, f, f, dX=torch.zeros(5, 16, device="cuda"))
    with pytest.raises(rov.RovError):
        rov.linear_xent(X, W, t, ignore_index=3)
    with pytest.raises(rov.RovError):
        rov.linear_xent(X, W, t, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(rov.RovError):
        rov.linear_xent_bwd(X, W, t, f, f, need_dX=False, need_dW=False)
