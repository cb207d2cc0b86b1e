"""The norms around a block against their formulas in 64 bits, and their gradients against automatic differentiation in
64 bits and against differences.

Tolerances.  Row sums run over at most 32 terms a thread and ten steps of a tree, so a mean of squares is off by less than
50 * 2^-24 of itself and its root by half of that; products and sums around it add a few 2^-24 each: together below 2^-18
of the terms' magnitudes (M below, formed with absolute values).  Gradients go through two such rows: 2^-17.  Column sums chain at most some 200
additions: 2^-16 of the sum of magnitudes.  A bf16 result is off by another 2^-8 of the value, an e4m3 result by 2^-4 of it or
half of its smallest step, 2^-10, times the scale.
"""
import pytest
import torch

from paper_2410_07531_amd import binding as rov

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


def make(rows, n, dtype, gates, post, pre, seed=0, backward=False):
    g = torch.Generator().manual_seed(seed + rows * 31 + n)
    r = lambda *s: torch.randn(*s, generator=g).to(DT[dtype]).cuda()
    d = dict(h=r(rows, n), w_post=(1 + 0.1 * r(n)) if post else None, w_pre=(1 + 0.1 * r(n)) if pre else None,
             gate=r(gates, n) if gates else None)
    d.update(dict(y=r(rows, n), dy=r(rows, n), dn=r(rows, n) if pre else None) if backward else dict(x=2 * r(rows, n)))
    return d


def f64(v):
    return None if v is None else v.double().cpu()


def rms(v):
    return v / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS)


def spread(gate, rows):
    return 1.0 if gate is None else gate.repeat_interleave(rows // gate.shape[0], 0)


def forward(d, xs, hs):
    x, h, wp, wn, g = (f64(d[k]) for k in ("x", "h", "w_post", "w_pre", "gate"))
    rows = x.shape[0]
    b = hs * spread(g, rows) * (h if wp is None else rms(h) * wp)
    y, mag = xs * x + b, abs(xs) * x.abs() + b.abs()
    if wn is None:
        return y, mag, None, None
    r = 1.0 / torch.sqrt((y * y).mean(-1, keepdim=True) + EPS)
    return y, mag, y * r * wn, (mag + y.abs()) * r * wn.abs()


def check(got, want, mag, dtype, rel):
    err = (got.double().cpu() - want).abs()
    tol = rel * mag + (2.0 ** -8 * want.abs() if dtype == "bf16" else 0.0)
    assert bool((err <= tol).all()), (float((err - tol).max()), float(err.max()))


SHAPES = [(1, 1), (3, 8), (5, 100), (2, 1001), (7, 512), (4, 1024), (9, 2816), (3, 4096), (2, 8192), (2, 8200), (1, 32768), (2, 30001)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,n", SHAPES)
@pytest.mark.parametrize("gates,post,pre", [(1, True, True), (0, False, True), (0, True, False), (-1, False, True)])
def test_forward(dtype, rows, n, gates, post, pre):
    print("norm fwd", dtype, rows, n, gates, post, pre, flush=True)
    d = make(rows, n, dtype, rows if gates < 0 else gates, post, pre)
    y, yn = rov.norm_residual(d["x"], d["h"], d["w_pre"], d["w_post"], d["gate"], x_scale=0.75, h_scale=0.5, eps=EPS)
    wy, my, wn, mn = forward(d, 0.75, 0.5)
    check(y, wy, my, dtype, 2.0 ** -18)
    assert (yn is None) == (wn is None)
    if pre:
        check(yn, wn, mn, dtype, 2.0 ** -18)


def test_forward_many_rows_with_shared_gates():
    d = make(3000, 1024, "bf16", 6, True, True)
    y, yn = rov.norm_residual(d["x"], d["h"], d["w_pre"], d["w_post"], d["gate"])
    wy, my, wn, mn = forward(d, 1.0, 1.0)
    check(y, wy, my, "bf16", 2.0 ** -18)
    check(yn, wn, mn, "bf16", 2.0 ** -18)


@pytest.mark.parametrize("n", [4096, 1001])
def test_forward_into_e4m3(n):
    d = make(5, n, "bf16", 0, True, True)
    scale = 0.02
    _, y8 = rov.norm_residual(d["x"], d["h"], d["w_pre"], d["w_post"], yn_fp8_scale=scale)
    want, mag = forward(d, 1.0, 1.0)[2:]
    got = y8.view(torch.float8_e4m3fn).double().cpu() * scale
    err = (got - want).abs()
    assert bool((err <= 2.0 ** -4 * want.abs() + 2.0 ** -10 * scale + 2.0 ** -17 * mag).all())


def test_forward_in_place_and_strided():
    d = make(6, 512, "bf16", 0, True, True)
    want = rov.norm_residual(d["x"], d["h"], d["w_pre"], d["w_post"])
    wide = torch.full((6, 1024), 3.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 256:768] = d["x"]
    x = wide[:, 256:768]
    h = d["h"].clone()
    y, yn = rov.norm_residual(x, h, d["w_pre"], d["w_post"], y=x, yn=h)
    assert torch.equal(y, want[0]) and torch.equal(yn, want[1])
    assert bool((wide[:, :256] == 3.0).all()) and bool((wide[:, 768:] == 3.0).all())
    # rows off 16 bytes take another kernel: the same values to a rounding
    odd = torch.empty(6, 515, dtype=torch.bfloat16, device="cuda")[:, 3:]
    odd.copy_(d["x"])
    y2, yn2 = rov.norm_residual(odd, d["h"], d["w_pre"], d["w_post"])
    wy, my, wn, mn = forward(d, 1.0, 1.0)
    check(y2, wy, my, "bf16", 2.0 ** -18)
    check(yn2, wn, mn, "bf16", 2.0 ** -18)


def test_rows_of_zeros_and_infinities_stay_apart():
    d = make(4, 256, "f32", 0, True, True)
    d["x"][1] = 0
    d["h"][1] = 0
    d["h"][2, 7] = float("inf")
    y, yn = rov.norm_residual(d["x"], d["h"], d["w_pre"], d["w_post"])
    assert bool((y[1] == 0).all()) and bool((yn[1] == 0).all()) and bool(torch.isnan(y[2, 7]))
    wy, my, wn, mn = forward(d, 1.0, 1.0)
    for r in (0, 3):
        check(yn[r:r + 1], wn[r:r + 1], mn[r:r + 1], "f32", 2.0 ** -18)


def gradients(d, xs, hs):
    """Gradients in float64 by automatic differentiation, and magnitudes for the tolerances by the formulas."""
    rows, n = d["dy"].shape if d["dy"] is not None else d["dn"].shape
    h, wp, wn, g = (None if d[k] is None else f64(d[k]).requires_grad_() for k in ("h", "w_post", "w_pre", "gate"))
    b = hs * spread(g, rows) * (h if wp is None else rms(h) * wp)
    x = ((f64(d["y"]) - b.detach()) / xs).requires_grad_()
    y = xs * x + b
    total = 0.0
    if d["dy"] is not None:
        total = total + (y * f64(d["dy"])).sum()
    if wn is not None:
        total = total + (rms(y) * wn * f64(d["dn"])).sum()
    total.backward()
    grad = lambda v: None if v is None else v.grad
    y, hd, a = y.detach(), h.detach(), (lambda v: 1.0 if v is None else v.detach().abs())
    mean = lambda v: v.mean(-1, keepdim=True)
    mg = 0.0 if d["dy"] is None else f64(d["dy"]).abs()
    M = {}
    if wn is not None:
        r = 1 / torch.sqrt(mean(y * y) + EPS)
        t = f64(d["dn"]).abs() * a(wn)
        mg = mg + r * t + y.abs() * r ** 3 * mean(y.abs() * t)
        M["w_pre"] = (f64(d["dn"]).abs() * y.abs() * r).sum(0)
    rh = 1.0 if wp is None else 1 / torch.sqrt(mean(hd * hd) + EPS)
    q = abs(hs) * spread(g, rows).abs().detach() * mg if g is not None else abs(hs) * mg
    t = q * a(wp)
    M["h"] = rh * t + (0.0 if wp is None else hd.abs() * rh ** 3 * mean(hd.abs() * t))
    M["x"] = abs(xs) * mg
    if wp is not None:
        M["w_post"] = (q * hd.abs() * rh).sum(0)
    if g is not None:
        M["gate"] = (abs(hs) * mg * rh * hd.abs() * a(wp)).reshape(g.shape[0], -1, n).sum(1)
    return dict(x=x.grad, h=h.grad, w_pre=grad(wn), w_post=grad(wp), gate=grad(g)), M


def check_gradients(d, got, xs, hs, dtype):
    want, M = gradients(d, xs, hs)
    for name, t in zip(("x", "h", "w_pre", "w_post", "gate"), got):
        assert (t is None) == (want[name] is None), name
        if t is None:
            continue
        print(" ", name, flush=True)
        sums = name not in ("x", "h")
        assert t.dtype == (torch.float32 if sums else DT[dtype])
        check(t.reshape(want[name].shape), want[name], M[name], "f32" if sums else dtype, 2.0 ** -16 if sums else 2.0 ** -17)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,n", SHAPES + [(130, 64), (1201, 72)])
@pytest.mark.parametrize("gates,post,pre", [(1, True, True), (0, False, True), (0, True, False), (-1, True, True), (-1, False, False)])
def test_backward(dtype, rows, n, gates, post, pre):
    print("norm bwd", dtype, rows, n, gates, post, pre, flush=True)
    d = make(rows, n, dtype, rows if gates < 0 else gates, post, pre, backward=True)
    got = rov.norm_residual_bwd(d["y"], d["h"], d["dy"], d["dn"], d["w_pre"], d["w_post"], d["gate"], x_scale=0.75, h_scale=0.5, eps=EPS)
    check_gradients(d, got, 0.75, 0.5, dtype)


@pytest.mark.parametrize("rows,gates", [(2400, 3), (5000, 2500), (4100, 4100), (2050, 1)])
def test_backward_shares_of_rows(rows, gates):
    # several workgroups a gate, several gates a workgroup, one gate a row
    d = make(rows, 256, "f32", gates, True, True, backward=True)
    kw = dict(x_scale=1.0, h_scale=0.5, eps=EPS)
    args = (d["y"], d["h"], d["dy"], d["dn"], d["w_pre"], d["w_post"], d["gate"])
    got = rov.norm_residual_bwd(*args, **kw)
    check_gradients(d, got, 1.0, 0.5, "f32")
    again = rov.norm_residual_bwd(*args, **kw)
    assert all(torch.equal(a, b) for a, b in zip(got, again))     # sums in a fixed order


def test_backward_without_dy_and_in_place():
    d = make(33, 512, "bf16", 0, True, True, backward=True)
    want = rov.norm_residual_bwd(d["y"], d["h"], d["dy"], d["dn"], d["w_pre"], d["w_post"])
    dy, dn = d["dy"].clone(), d["dn"].clone()
    got = rov.norm_residual_bwd(d["y"], d["h"], dy, dn, d["w_pre"], d["w_post"], dx=dy, dh=dn)
    assert all(a is b is None or torch.equal(a, b) for a, b in zip(got, want))
    d["dy"] = None
    got = rov.norm_residual_bwd(d["y"], d["h"], None, d["dn"], d["w_pre"], d["w_post"])
    check_gradients(d, got, 1.0, 1.0, "bf16")


def test_gradient_against_differences():
    # central differences of the library's own forward pass in fp32 along random directions
    d = make(9, 320, "f32", 3, True, True)
    g = torch.Generator().manual_seed(9)
    u = [torch.randn(9, 320, generator=g).cuda().double() for _ in range(2)]
    names = ("x", "h", "w_pre", "w_post", "gate")

    def loss(v):
        y, yn = rov.norm_residual(v["x"], v["h"], v["w_pre"], v["w_post"], v["gate"], x_scale=0.9, h_scale=0.5, eps=EPS)
        return float((y.double() * u[0]).sum() + (yn.double() * u[1]).sum()), y

    y = loss(d)[1]
    got = dict(zip(names, rov.norm_residual_bwd(y, d["h"], u[0].float(), u[1].float(), d["w_pre"], d["w_post"], d["gate"], x_scale=0.9,
                                                h_scale=0.5, eps=EPS)))
    for name in names:
        direction = torch.randn(d[name].shape, generator=g).cuda()
        step = 1e-2
        plus, minus = (loss({**d, name: d[name] + s * direction})[0] for s in (step, -step))
        slope = float((got[name].double() * direction.double()).sum())
        # the forward's fp32 rounding over the step (5760 outputs of size about 1 at 2^-22, random) and the third-order term
        assert abs((plus - minus) / (2 * step) - slope) <= 2.0 ** -22 * 5760 ** 0.5 * 4 / step + 2e-3 * (abs(slope) + 5760 ** 0.5), name


def test_stream_and_graph():
    d = make(40, 1024, "bf16", 1, True, True, backward=True)
    d["x"] = d["y"]
    want = rov.norm_residual_bwd(d["y"], d["h"], d["dy"], d["dn"], d["w_pre"], d["w_post"], d["gate"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = rov.norm_residual_bwd(d["y"], d["h"], d["dy"], d["dn"], d["w_pre"], d["w_post"], d["gate"], stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fwd = rov.norm_residual(d["x"], d["h"], d["w_pre"], d["w_post"], d["gate"])
        bwd = rov.norm_residual_bwd(fwd[0], d["h"], d["dy"], d["dn"], d["w_pre"], d["w_post"], d["gate"])
    for i in range(3):
        d["h"].mul_(1.25)
        graph.replay()
        torch.cuda.synchronize()
        f = rov.norm_residual(d["x"], d["h"], d["w_pre"], d["w_post"], d["gate"])
        b = rov.norm_residual_bwd(f[0], d["h"], d["dy"], d["dn"], d["w_pre"], d["w_post"], d["gate"])
        assert all(torch.equal(a, c) for a, c in zip(fwd + bwd, f + b)), i


def test_refusals_in_the_binding():
    x = torch.zeros(4, 64, device="cuda")
    for bad in (dict(h=torch.zeros(4, 32, device="cuda")), dict(h=x, w_pre=torch.zeros(63, device="cuda")), dict(h=x, gate=torch.zeros(3, 64, device="cuda")),
                dict(h=x.cpu()), dict(h=x.t().contiguous().t()), dict(h=x, y=torch.zeros(5, 64, device="cuda"))):
        with pytest.raises(ValueError):
            rov.norm_residual(x, **bad)
    with pytest.raises(TypeError):
        rov.norm_residual(x, x.to(torch.bfloat16))
    for empty in (torch.zeros(0, 64, device="cuda"), torch.zeros(4, 0, device="cuda"), torch.zeros((), device="cuda")):
        with pytest.raises(ValueError):
            rov.norm_residual(empty, empty)
        with pytest.raises(ValueError):
            rov.norm_residual_bwd(empty, empty, empty)
    with pytest.raises(ValueError):
        rov.norm_residual_bwd(x, x, None)
    with pytest.raises(rov.RovError):
        rov.norm_residual_bwd(x, x, x, None, w_pre=x[0].contiguous())
    with pytest.raises(rov.RovError):
        rov.norm_residual_bwd(x, x, x, x, w_pre=x[0].contiguous(), workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))


# ---- rows of no whole 16-byte pieces, longer than those that move element by element
RAGGED = [(3, 1025), (5, 1501), (2, 2050), (3, 4099), (2, 8191), (2, 8201), (2, 16381), (1, 32767), (67, 1030)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,n", RAGGED)
@pytest.mark.parametrize("gates,post", [(1, True), (-1, True), (0, False)])
def test_ragged_rows(dtype, rows, n, gates, post):
    print("norm ragged", dtype, rows, n, gates, post, flush=True)
    d = make(rows, n, dtype, rows if gates < 0 else gates, post, True)
    y, yn = rov.norm_residual(d["x"], d["h"], d["w_pre"], d["w_post"], d["gate"], x_scale=0.75, h_scale=0.5, eps=EPS)
    wy, my, wn, mn = forward(d, 0.75, 0.5)
    check(y, wy, my, dtype, 2.0 ** -18)
    check(yn, wn, mn, dtype, 2.0 ** -18)
    d = make(rows, n, dtype, rows if gates < 0 else gates, post, True, backward=True)
    got = rov.norm_residual_bwd(d["y"], d["h"], d["dy"], d["dn"], d["w_pre"], d["w_post"], d["gate"], x_scale=0.75, h_scale=0.5, eps=EPS)
    check_gradients(d, got, 0.75, 0.5, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [512, 1027, 4096, 4101, 9000])
def test_any_stride_and_address(dtype, n):
    # in place inside wider rows that start off 16 bytes: the bits of dense rows, and what lies around them stays
    rows = 4
    d = make(rows, n, dtype, 2, True, True, seed=9)
    b = make(rows, n, dtype, 2, True, True, seed=9, backward=True)

    def inside(t):
        wide = torch.full((rows, n + 7), 3.0, dtype=DT[dtype], device="cuda")
        wide[:, 3:3 + n] = t
        return wide, wide[:, 3:3 + n]

    want = rov.norm_residual(d["x"], d["h"], d["w_pre"], d["w_post"], d["gate"])
    (wx, x), (wh, h) = inside(d["x"]), inside(d["h"])
    got = rov.norm_residual(x, h, d["w_pre"], d["w_post"], d["gate"], y=x, yn=h)
    want_b = rov.norm_residual_bwd(b["y"], b["h"], b["dy"], b["dn"], b["w_pre"], b["w_post"], b["gate"])
    (wd, dy), (we, e) = inside(b["dy"]), inside(b["h"])
    got_b = rov.norm_residual_bwd(inside(b["y"])[1], e, dy, inside(b["dn"])[1], b["w_pre"], b["w_post"], b["gate"], dx=dy, dh=e)
    assert all(torch.equal(a, c) for a, c in zip(want, got)) and all(torch.equal(a, c) for a, c in zip(want_b, got_b))
    for wide in (wx, wh, wd, we):
        assert bool((wide[:, :3] == 3.0).all()) and bool((wide[:, 3 + n:] == 3.0).all())


def test_ragged_rows_into_e4m3_behind_a_guard():
    d = make(5, 1501, "bf16", 0, True, True)
    out = torch.full((5, 1505), 7, dtype=torch.uint8, device="cuda")
    rov.norm_residual(d["x"], d["h"], d["w_pre"], d["w_post"], yn=out[:, :1501], yn_fp8_scale=0.02)
    want, mag = forward(d, 1.0, 1.0)[2:]
    err = (out[:, :1501].contiguous().view(torch.float8_e4m3fn).double().cpu() * 0.02 - want).abs()
    assert bool((err <= 2.0 ** -4 * want.abs() + 2.0 ** -10 * 0.02 + 2.0 ** -17 * mag).all()) and bool((out[:, 1501:] == 7).all())
