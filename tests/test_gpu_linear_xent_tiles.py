"""Loss over the vocabulary with softmaxes that are not one-hot, at sizes where a workgroup takes one tile or several, and the proof on the CPU
that the comparison would show a wrong tile.

Inputs: rows of W of length S, X normal plus the multiple of the target's row that adds LEAN to its logit, so that a row's logits spread by about S
and its target has a probability around a half of what LEAN makes of it: from 0.02 to 0.9 over the rows.
Tolerances: element by element those of test_gpu_linear_xent.py.  They are worst cases, so a norm is taken too: roundings to bf16 are independent and
each at most half a step, 2^-8 of its value, evenly spread within it, so a root mean square of at most 2^-8 / sqrt(3): the squared norm
of the errors is (2^-16 / 3) times the sum of squares of the results and of all terms whose factor was rounded (G for dX; G and, by another rounding, X
for dW), within 1.3 times its root for more than a thousand results; the terms in fp32 add 2^-12 of that.
"""
import math

import pytest
import torch

import test_gpu_linear_xent as L
from paper_2410_07531_amd import binding as rov

gpu = pytest.mark.gpu
S = 1.5

# rows, vocabulary, K, columns of a piece, products whose workgroups take several tiles (loss, gradients): 1 and 2 logits, 4 dX, 8 dW
WALKS = [(300, 51000, 128, 0, 1, 2),        # two slots of k: the next tile is aimed at in the first
         (600, 34000, 192, 0, 1, 2),        # three slots
         (300, 51000, 136, 0, 1, 2),        # the last slot a part
         (300, 51000, 264, 0, 1, 2 | 8),
         (130, 51000, 264, 0, 0, 8),        # dW over two slots and a part
         (500, 51000, 300, 0, 1, 2 | 8),    # packed operands
         (1000, 33200, 264, 0, 1, 2),       # two full rounds of tiles and a rest of narrower ones
         (150, 66000, 264, 0, 0, 8),        # the same for dW
         (16, 131073, 136, 0, 1, 2),        # few rows, whose dW has a kernel of its own
         (51000, 300, 264, 0, 1, 2 | 4),    # dX at once
         (51000, 600, 264, 256, 1, 4),      # dX summed over pieces
         (66000, 300, 512, 0, 1, 2 | 4)]    # rows: full rounds and a rest
PLAIN = [s for s in L.SIZES if s[1] >= 200]
CASES = PLAIN + [s[:4] for s in WALKS]


def make(M, V, K, dtype, seed=0, ignored=0.2):
    g = torch.Generator().manual_seed(seed + 1000 * M + V + K)
    W = (torch.randn(V, K, generator=g) * S / K ** 0.5).to(L.DT[dtype])
    t = torch.randint(0, V, (M,), generator=g)
    lean = math.log(V) + S * S / 2 - 1.0      # a probability of 1 / (1 + e) where the row's other logits are as expected
    w = W[t].float()
    X = (torch.randn(M, K, generator=g) + lean * w / (w * w).sum(1, keepdim=True).clamp(min=0.1)).to(L.DT[dtype])
    t[torch.rand(M, generator=g) < ignored] = -100
    return X, W, t, torch.rand(M, generator=g) + 0.5


def answer(X, W, t, dloss):
    """Reference results and tolerances, the gradients' norms that errors may have, and the terms to plant mistakes with."""
    r = L.reference(X, W, t, dloss)
    x, w, keep = X.double(), W.double(), t != -100
    P = torch.softmax(x @ w.t(), 1)
    a = dloss.double() * keep
    at = torch.where(keep, t, torch.zeros_like(t))[:, None]
    G = (P * a[:, None]).scatter_add(1, at, -a[:, None])
    G2, x2 = G.square(), x.square()
    half = 2.0 ** -16 / 3
    r["nX"] = 1.3 * float((half * (r["dX"].square().sum() + (G2.sum(0) @ w.square()).sum())).sqrt()) + 2.0 ** -12 * float(r["dX"].norm())
    r["nW"] = 1.3 * float((half * (r["dW"].square().sum() + 2 * (G2.sum(1) @ x2).sum())).sqrt()) + 2.0 ** -12 * float(r["dW"].norm())
    return r, P, G, a


def faults(r, loss, lse, dX=None, dW=None, rows=0):
    """What of the results is outside its tolerances."""
    got = []
    for name, v, tol in (("loss", loss, "tol"), ("lse", lse, "tol"), ("dX", dX, "tX"), ("dW", dW, "tW")):
        if v is None:
            continue
        err = (v.double() - r[name]).abs()
        if not bool((err <= r[tol]).all()):
            got.append(name)
        elif tol != "tol" and rows >= 100 and not float(err.norm()) <= r["n" + name[1]]:
            got.append("norm of " + name)
    return got


@pytest.mark.parametrize("M,V,K", sorted({s[:3] for s in CASES if s[0] >= 17}))
def test_wrong_answers_fall_outside(M, V, K):
    # the tolerances are those of bf16, the wider ones; results in 64 bits with a mistake in them
    X, W, t, dloss = make(M, V, K, "bf16")
    r, P, G, a = answer(X, W, t, dloss)
    x, w, keep = X.double(), W.double(), t != -100
    z_t = r["lse"] - torch.where(keep, r["loss"], torch.zeros_like(r["loss"]))
    first = int(keep.nonzero()[0])
    tile = slice(first // 256 * 256, first // 256 * 256 + 256), slice(int(t[first]) // 256 * 256, int(t[first]) // 256 * 256 + 256)   # rows, columns
    assert faults(r, r["loss"], r["lse"], r["dX"], r["dW"], M) == []

    def shows(what, *names, **wrong):
        found = faults(r, wrong.get("loss", r["loss"]), wrong.get("lse", r["lse"]), wrong.get("dX", r["dX"]), wrong.get("dW", r["dW"]), M)
        assert all(any(n in f for f in found) for n in names), (what, found)

    def without(what, rows, cols):
        # this part of the logits left out of the sums, of G, of the results' rows
        left = 1.0 - P[rows, cols].sum(1)
        lse = r["lse"].clone()
        lse[rows] += torch.log(left.clamp(min=1e-300))
        g = G.clone()
        g[rows, cols] = 0
        shows(what, "lse", "dX", "dW", lse=lse, dX=g @ w, dW=g.t() @ (x * keep[:, None]))

    shows("no gradients", "dX", "dW", dX=torch.zeros_like(r["dX"]), dW=torch.zeros_like(r["dW"]))
    shows("the target's column alone", "lse", "loss", lse=z_t, loss=torch.zeros_like(z_t))
    one_hot = torch.zeros_like(G).scatter_(1, t.clamp(min=0)[:, None], -a[:, None])
    shows("no softmax term", "dX", "dW", dX=one_hot @ w, dW=one_hot.t() @ x)
    without("a tile", *tile)
    without("the first half of the vocabulary", slice(0, M), slice(0, V // 2))
    for name, v, at in (("dX", r["dX"], (tile[0], slice(0, 256))), ("dW", r["dW"], (tile[1], slice(0, 256)))):
        bad = v.clone()
        bad[at] = 0
        shows("a tile not written", name, **{name: bad})
    g = G.clone()
    g[first // 64 * 64:first // 64 * 64 + 64] = 0
    shows("64 rows of dW's sums", "dW", dW=g.t() @ (x * keep[:, None]))
    g = G.clone()
    g[:, int(t[first]) // 64 * 64:int(t[first]) // 64 * 64 + 64] = 0
    shows("64 columns of dX's sums", "dX", dX=g @ w)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,V,K,piece", PLAIN)
def test_loss_and_gradients(dtype, M, V, K, piece):
    print("xent", dtype, M, V, K, piece, flush=True)
    X, W, t, dloss = (v.cuda() for v in make(M, V, K, dtype))
    r = answer(X, W, t, dloss)[0]
    loss, lse = rov.linear_xent(X, W, t, vocab_piece=piece)
    dX, dW = rov.linear_xent_bwd(X, W, t, lse, dloss, vocab_piece=piece)
    assert faults(r, loss, lse, dX, dW, M) == []


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_with_one_gradient_or_none(dtype):
    # a row's factor is dloss, or the sum where dloss is next to nothing beside it: rows with dlse alone, nothing, a sum of zero, a dloss of 2^-30
    M, V, K = 300, 1300, 264
    X, W, t, dloss = (v.cuda() for v in make(M, V, K, dtype, ignored=0.1))
    dlse = 0.3 * torch.randn(M, generator=torch.Generator().manual_seed(3)).cuda()
    dloss[0::5] = 0
    dloss[1::10], dlse[1::10] = 0, 0
    dlse[2::5] = -dloss[2::5]
    dloss[3::5] *= 2.0 ** -30
    r = L.reference(X, W, t, dloss, dlse)
    _, lse = rov.linear_xent(X, W, t)
    dX, dW = rov.linear_xent_bwd(X, W, t, lse, dloss, dlse)
    L.close(dX, r["dX"], r["tX"], "dX")
    L.close(dW, r["dW"], r["tW"], "dW")
    assert bool((dX[1::10] == 0).all())


def test_which_products_walk_over_tiles():
    # (256 compute units: the chip's, and what the library goes by without one)
    for M, V, K, piece, forward, backward in WALKS:
        assert rov.linear_xent_walks(M, V, K, False, piece) == forward and rov.linear_xent_walks(M, V, K, True, piece) == backward, (M, V, K, piece)
    assert rov.linear_xent_walks(8192, 131072, 4096, True) == 2 | 4 | 8
    for M, V, K, piece in L.SIZES:      # those of the other tests have a tile a workgroup
        assert rov.linear_xent_walks(M, V, K, False, piece) == rov.linear_xent_walks(M, V, K, True, piece) == 0
    for bad in ((0, 10, 8), (4, -1, 8), (4, 10, 0)):
        with pytest.raises(rov.RovError) as e:
            rov.linear_xent_walks(*bad)
        assert e.value.code == rov.ERR_INVALID


@gpu
@pytest.mark.parametrize("M,V,K,piece,forward,backward", WALKS)
def test_a_workgroup_with_several_tiles(M, V, K, piece, forward, backward):
    print("xent walk", M, V, K, piece, flush=True)
    assert rov.linear_xent_walks(M, V, K, False, piece) == forward and rov.linear_xent_walks(M, V, K, True, piece) == backward
    X, W, t, dloss = (v.cuda() for v in make(M, V, K, "bf16"))
    r = answer(X, W, t, dloss)[0]
    loss, lse = rov.linear_xent(X, W, t, vocab_piece=piece)
    dX, dW = rov.linear_xent_bwd(X, W, t, lse, dloss, vocab_piece=piece)
    assert faults(r, loss, lse, dX, dW, M) == []
    for _ in range(3):      # the same bits each time, whatever ran before
        rov.linear_xent_bwd(X.flip(0), W, t, lse, dloss, vocab_piece=piece)
        again = rov.linear_xent(X, W, t, vocab_piece=piece) + rov.linear_xent_bwd(X, W, t, lse, dloss, vocab_piece=piece)
        assert all(torch.equal(a, b) for a, b in zip(again, (loss, lse, dX, dW)))


@gpu
def test_several_tiles_captured_and_beside_another_call():
    # a graph replayed between eager calls, and two streams that work on different inputs at once, each with its own workspace
    M, V, K = 300, 51000, 264
    X, W, t, dloss = (v.cuda() for v in make(M, V, K, "bf16"))
    X2, t2 = X.flip(0).contiguous(), t.flip(0).contiguous()

    def both(X, t, stream=None):
        loss, lse = rov.linear_xent(X, W, t, stream=stream)
        return (loss, lse) + rov.linear_xent_bwd(X, W, t, lse, dloss, stream=stream)

    want, want2 = both(X, t), both(X2, t2)
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        a, b = both(X, t, one), both(X2, t2, two)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a + b, want + want2))
    held, at = X.clone(), t.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both(held, at)
    for x, y, w in ((X2, t2, want2), (X, t, want), (X2, t2, want2)):
        held.copy_(x)
        at.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(got, w))
        assert all(torch.equal(u, v) for u, v in zip(both(X, t), want))
