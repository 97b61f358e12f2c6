"""Softmax loss and its gradient (ivfr_softmax_*) against the definition in 64 bits.

Tolerances, derived.  A score is a sum of d products: fp32 accumulation makes it wrong by at most (d + 8) 2^-24 of sum |x w| (fp32
inputs: their three-part split neglects 2^-22 more), the epilogue by 2^-22 of it.  A loss is the difference of two numbers that are wrong
by as much each, and the statistics add 2^-20 of one plus the loss.  e is wrong by its rounding to the type (2^-9, 2^-12, 2^-24 of itself) and by
the scores' error times the probability; a gradient by the sums of both over the other operand, by the accumulation of as many terms, and by its own rounding."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def make(n, v, d, dtype, seed=0, offset=False, ignored=False):
    g = torch.Generator(device="cuda").manual_seed(1000 * seed + n + 7 * v + 13 * d)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    w = r(v, d)
    targets = torch.randint(0, v, (n,), generator=g, device="cuda")
    x = 2 * r(n, d) + w[targets] * (4 / math.sqrt(d))
    weight = (0.25 + torch.rand(n, generator=g, device="cuda")) / max(n, 1) * torch.where(torch.rand(n, generator=g, device="cuda") < 0.2, -1.0, 1.0)
    o = None
    if offset:
        o = r(v)
        if v > 2:
            o[torch.rand(v, generator=g, device="cuda") < 0.2] = -math.inf
    if ignored:
        targets[torch.rand(n, generator=g, device="cuda") < 0.3] = -1
    return x.to(TYPES[dtype]), w.to(TYPES[dtype]), targets, weight, 1 / math.sqrt(d), o


def reference(x, w, targets, weight, scale, offset):
    """(loss, lse, dx, dw) and bounds on the scores' error and on the gradients', all float64."""
    x, w = x.double(), w.double()
    n, v = x.shape[0], w.shape[0]
    z = torch.mm(x, w.t()) * scale
    size = torch.mm(x.abs(), w.abs().t()) * abs(scale)
    if offset is not None:
        z = z + offset.double()
        out = torch.isinf(offset)
        z[:, out] = -math.inf
        size = size + torch.where(out, 0.0, offset.double()).abs()
        size[:, out] = 0
    has = targets >= 0
    t = targets.clamp(0, v - 1)
    lse = torch.logsumexp(z, 1)
    zt = z.gather(1, t[:, None])[:, 0]
    loss = torch.where(has, torch.where(torch.isinf(zt), math.inf, lse - zt), 0.0)
    p = torch.where(torch.isinf(z), 0.0, torch.exp(z - lse[:, None]))
    hot = torch.zeros_like(p)
    hot.scatter_(1, t[:, None], 1.0)
    hot = torch.where(torch.isinf(z), 0.0, hot)
    g = torch.where(has, weight.double(), 0.0)[:, None]
    e = g * (p - hot)
    return loss, lse, scale * torch.mm(e, w), scale * torch.mm(e.t(), x), size, p * g.abs(), e.abs()


def bounds(dtype, x, w, scale, size, pg, e):
    d = x.shape[1]
    ez = size * ((d + 8) * 2.0 ** -24 + 2.0 ** -22 + (2.0 ** -22 if dtype == "f32" else 0))
    score = ez.amax(1)
    # the statistics: every probability is wrong by its score's error and the row's largest, and by 2^-20 of itself
    de = e * UNIT[dtype] + pg * (ez + score[:, None] + 2.0 ** -20) * 1.01
    aw, ax = w.double().abs(), x.double().abs()
    u, s = UNIT[dtype], abs(scale)
    n, v = e.shape
    tiny = 2.0 ** -24 if dtype == "f16" else 2.0 ** -126
    bx = s * torch.mm(de, aw) + s * torch.mm(e, aw) * (v + 64) * 2.0 ** -24
    bw = s * torch.mm(de.t(), ax) + s * torch.mm(e.t(), ax) * (n + 64) * 2.0 ** -24
    return score, lambda ref: bx + u * ref.abs() + tiny, lambda ref: bw + u * ref.abs() + tiny


def check(dtype, args, outs=None):
    import paper_1102_3828_amd as pkg
    x, w, targets, weight, scale, offset = args
    loss, lse = pkg.softmax_loss(x, w, targets, scale=scale, offset=offset)
    loss2, dx, dw = pkg.softmax_loss_grad(x, w, targets, weight, scale=scale, offset=offset)
    rl, rs, rx, rw, size, pg, e = reference(*args)
    score, bx, bw = bounds(dtype, x, w, scale, size, pg, e)
    inf = torch.isinf(rl)
    assert torch.equal(torch.isinf(loss) & (loss > 0), inf) and torch.equal(torch.isinf(loss2) & (loss2 > 0), inf)
    tol = 2 * score + 2.0 ** -20 * (1 + rl.abs()) + 2.0 ** -23 * rs.abs()
    for l in (loss, loss2):
        worst = ((l.double() - rl).abs()[~inf] / tol[~inf])
        assert worst.numel() == 0 or worst.max() <= 1, worst.max()
    live = ~torch.isinf(rs)
    assert torch.equal(torch.isinf(lse) & (lse < 0), ~live)
    worst = (lse.double() - rs).abs()[live] / (score + 2.0 ** -20 * (1 + rs.abs()))[live]
    assert worst.numel() == 0 or worst.max() <= 1, worst.max()
    assert dx.dtype == x.dtype and dw.dtype == w.dtype and dx.shape == x.shape and dw.shape == w.shape
    assert ((dx.double() - rx).abs() <= bx(rx)).all(), ((dx.double() - rx).abs() / bx(rx)).max()
    assert ((dw.double() - rw).abs() <= bw(rw)).all(), ((dw.double() - rw).abs() / bw(rw)).max()
    return loss, lse, dx, dw


SHAPES = [(1, 1, 1), (1, 2, 3), (3, 1, 8), (2, 500, 32), (17, 1000, 128), (16, 257, 64), (33, 255, 64), (64, 300, 200), (65, 300, 33),
          (130, 1031, 96), (300, 513, 77), (1, 4097, 2048), (257, 2050, 40), (600, 90, 256), (1000, 33, 130)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("n,v,d", SHAPES)
def test_loss_and_gradient(n, v, d, dtype):
    check(dtype, make(n, v, d, dtype))


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("n,v,d", [(1, 7, 5), (40, 600, 64), (300, 1030, 100), (129, 2500, 192)])
def test_left_out_vectors_and_rows_without_target(n, v, d, dtype):
    """Removed vectors hold NaN, rows without a target too: neither shows in anything but such a row's lse."""
    x, w, t, g, s, o = make(n, v, d, dtype, offset=True, ignored=True)
    loss, lse, dx, dw = check(dtype, (x, w, t, g, s, o))
    import paper_1102_3828_amd as pkg
    w2, x2 = w.clone(), x.clone()
    w2[torch.isinf(o)] = math.nan
    x2[t < 0] = math.nan
    loss2, dx2, dw2 = pkg.softmax_loss_grad(x2, w2, t, g, scale=s, offset=o)
    l3, s3 = pkg.softmax_loss(x2, w2, t, scale=s, offset=o)
    assert torch.equal(loss, loss2) and torch.equal(dx, dx2) and torch.equal(dw, dw2)
    assert torch.equal(l3, loss) and torch.equal(s3[t >= 0], lse[t >= 0])
    assert (dw[torch.isinf(o)] == 0).all() and (dx[t < 0] == 0).all() and (loss[t < 0] == 0).all()


@pytest.mark.parametrize("dtype", list(TYPES))
def test_everything_left_out(dtype):
    import paper_1102_3828_amd as pkg
    x, w, t, g, s, _ = make(9, 300, 64, dtype)
    o = torch.full((300,), -math.inf, device="cuda")
    loss, lse = pkg.softmax_loss(x, w, t, scale=s, offset=o)
    assert (loss == math.inf).all() and (lse == -math.inf).all()
    loss, dx, dw = pkg.softmax_loss_grad(x, w, t, g, scale=s, offset=o)
    assert (loss == math.inf).all() and (dx == 0).all() and (dw == 0).all()


def test_what_is_not_a_number_shows():
    import paper_1102_3828_amd as pkg
    x, w, t, g, s, _ = make(50, 400, 64, "bf16")
    t2 = t.clone()
    t2[7] = 400                                   # no such vector
    loss, dx, dw = pkg.softmax_loss_grad(x, w, t2, g, scale=s)
    keep = torch.arange(50, device="cuda") != 7
    good, gx, _ = pkg.softmax_loss_grad(x, w, t, g, scale=s)
    assert loss[7].isnan() and torch.equal(loss[keep], good[keep]) and dx[7].isnan().all() and torch.equal(dx[keep], gx[keep]) and dw.isnan().all()
    x2 = x.clone()
    x2[3, 5] = math.nan
    loss, lse = pkg.softmax_loss(x2, w, t, scale=s)
    keep = torch.arange(50, device="cuda") != 3
    assert loss[3].isnan() and lse[3].isnan() and torch.equal(loss[keep], good[keep])


@pytest.mark.parametrize("dtype", list(TYPES))
def test_scores_of_any_size(dtype):
    """Scores in the hundreds, of either sign: the maximum keeps the exponentials in range.  Probabilities of one leave a gradient of p - 1
    that is small, and formed before it is rounded."""
    x, w, t, g, s, _ = make(70, 700, 128, dtype)
    check(dtype, (x, w, t, g, s * 60, None))
    check(dtype, (x, w, t, g, -s * 60, None))
    check(dtype, (x, w, t, g, 0.0, None))


@pytest.mark.parametrize("dtype", list(TYPES))
def test_rows_with_strides_and_alignment(dtype):
    import paper_1102_3828_amd as pkg
    n, v, d = 45, 310, 64
    x, w, t, g, s, o = make(n, v, d, dtype, offset=True)
    ref = pkg.softmax_loss_grad(x, w, t, g, scale=s, offset=o)
    ref_s = pkg.softmax_loss(x, w, t, scale=s, offset=o)
    for shift, pad in ((0, 8), (1, 0), (3, 5), (0, 1)):
        def spread(a):
            buf = torch.full((a.shape[0] * (d + pad) + shift + 8,), math.nan, dtype=a.dtype, device="cuda")
            view = buf[shift:shift + a.shape[0] * (d + pad)].view(a.shape[0], d + pad)[:, :d]
            view.copy_(a)
            return view
        got = pkg.softmax_loss_grad(spread(x), spread(w), t.to(torch.int32), g, scale=s, offset=o)
        assert all(torch.equal(a, b) for a, b in zip(got, ref)), (shift, pad)
        got = pkg.softmax_loss(spread(x), spread(w), t, scale=s, offset=o)
        assert all(torch.equal(a, b) for a, b in zip(got, ref_s)), (shift, pad)
    got = pkg.softmax_loss_grad(x.t().contiguous().t(), w.t().contiguous().t(), t, g, scale=s, offset=o)
    assert all(torch.equal(a, b) for a, b in zip(got, ref))


def test_many_pieces():
    """More of e than is formed at a time: several pieces of the vectors, the last one narrower."""
    check("bf16", make(4100, 140003, 32, "bf16"))


@pytest.mark.parametrize("dtype", list(TYPES))
def test_same_bits_with_statistics_given_and_on_another_stream(dtype):
    import paper_1102_3828_amd as pkg
    x, w, t, g, s, o = make(200, 3000, 96, dtype, offset=True, ignored=True)
    loss, dx, dw = pkg.softmax_loss_grad(x, w, t, g, scale=s, offset=o)
    l, lse = pkg.softmax_loss(x, w, t, scale=s, offset=o)
    none, dx2, dw2 = pkg.softmax_loss_grad(x, w, t, g, scale=s, offset=o, lse=lse)
    assert none is None and torch.equal(l, loss) and torch.equal(dx, dx2) and torch.equal(dw, dw2)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = pkg.softmax_loss_grad(x, w, t, g, scale=s, offset=o, stream=side.cuda_stream)
    with torch.cuda.stream(side):
        got2 = pkg.softmax_loss_grad(x, w, t, g, scale=s, offset=o)
    side.synchronize()
    for a, b, c in zip(got, got2, (loss, dx, dw)):
        assert torch.equal(a, c) and torch.equal(b, c)


def test_captured_in_a_graph():
    import paper_1102_3828_amd as pkg
    x, w, t, g, s, o = make(100, 900, 64, "f16", offset=True)
    pkg.softmax_loss_grad(x, w, t, g, scale=s, offset=o)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = pkg.softmax_loss_grad(x, w, t, g, scale=s, offset=o)
    for seed in range(4):
        nx, nw, nt, ng, _, no = make(100, 900, 64, "f16", seed=seed, offset=True)
        for a, b in ((x, nx), (w, nw), (t, nt), (g, ng), (o, no)):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        ref = pkg.softmax_loss_grad(nx, nw, nt, ng, scale=s, offset=no)
        assert all(torch.equal(a, b) for a, b in zip(out, ref)), seed


def test_no_rows():
    import paper_1102_3828_amd as pkg
    for dtype in TYPES.values():
        x, w = torch.empty((0, 37), dtype=dtype, device="cuda"), torch.randn((51, 37), device="cuda").to(dtype)
        t = torch.empty((0,), dtype=torch.int64, device="cuda")
        loss, lse = pkg.softmax_loss(x, w, t)
        assert loss.shape == lse.shape == (0,)
        loss, dx, dw = pkg.softmax_loss_grad(x, w, t, torch.empty(0, device="cuda"))
        assert loss.shape == (0,) and dx.shape == (0, 37) and dw.shape == w.shape and (dw == 0).all()


def test_gradient_against_differences():
    """The loss itself, at two points along a direction: (f(+h) - f(-h)) / 2 h against the gradient's component.  With fp32 losses of about 2^3, wrong
    by some 2^-19 each, and h = 2^-5 of unit directions: an error of 2^-14 from rounding and of h^2 from the third derivative (scores' slopes below one)."""
    import paper_1102_3828_amd as pkg
    x, w, t, g, s, o = make(12, 60, 24, "f32", offset=True, ignored=True)
    t = torch.where((t >= 0) & torch.isinf(o[t.clamp(min=0)]), int(torch.nonzero(~torch.isinf(o))[0]), t)
    one = torch.ones_like(g)
    _, dx, dw = pkg.softmax_loss_grad(x, w, t, one, scale=s, offset=o)
    gen = torch.Generator(device="cuda").manual_seed(3)
    h = 2.0 ** -5
    total = lambda a, b: pkg.softmax_loss(a, b, t, scale=s, offset=o)[0].double().sum().item()
    for _ in range(6):
        ux, uw = torch.randn(x.shape, generator=gen, device="cuda"), torch.randn(w.shape, generator=gen, device="cuda")
        ux, uw = ux / ux.norm(), uw / uw.norm()
        for grad, f in ((dx * ux, lambda a: total(x + a * ux, w)), (dw * uw, lambda a: total(x, w + a * uw))):
            slope = (f(h) - f(-h)) / (2 * h)
            assert abs(slope - grad.double().sum().item()) <= 12 * 2.0 ** -14 + 12 * h * h, (slope, grad.sum())


def test_autograd():
    import paper_1102_3828_amd as pkg
    x, w, t, g, s, o = make(30, 200, 48, "bf16", offset=True, ignored=True)
    x.requires_grad_(True)
    w.requires_grad_(True)
    loss = pkg.SoftmaxLoss.apply(x, w, t, s, o)
    live = torch.isfinite(loss)
    torch.where(live, loss * g, 0.0).sum().backward()
    ref = pkg.softmax_loss_grad(x.detach(), w.detach(), t, torch.where(live, g, 0.0), scale=s, offset=o)
    assert torch.equal(x.grad, ref[1]) and torch.equal(w.grad, ref[2]) and torch.equal(loss.detach(), ref[0])


def test_refusals():
    import paper_1102_3828_amd as pkg
    import ctypes
    x, w, t, g, s, o = make(10, 20, 16, "bf16", offset=True)
    for bad in (lambda: pkg.softmax_loss(x, w.float(), t), lambda: pkg.softmax_loss(x, w[:, :8], t), lambda: pkg.softmax_loss(x, w, t[:5]),
                lambda: pkg.softmax_loss(x.double(), w.double(), t), lambda: pkg.softmax_loss(x, w, t.float()),
                lambda: pkg.softmax_loss(x, w, t, offset=o[:3]), lambda: pkg.softmax_loss(x, w, t, offset=o.double()),
                lambda: pkg.softmax_loss(x[0], w, t), lambda: pkg.softmax_loss(x.cpu(), w, t),
                lambda: pkg.softmax_loss_grad(x, w, t, g[:3]), lambda: pkg.softmax_loss_grad(x, w, t, g.half()),
                lambda: pkg.softmax_loss_grad(x, w, t, g, lse=g[:2])):
        with pytest.raises((ValueError, RuntimeError)):
            bad()
    with pytest.raises(pkg.IvfrError) as err:
        pkg.softmax_loss(x, w, t, scale=math.inf)
    assert err.value.code == pkg.binding.ERR_INVALID_ARG
    with pytest.raises(pkg.IvfrError):
        pkg.softmax_loss(x, w[:0], t)
    a = pkg.binding.SoftmaxArgs(10, 20, 16, 2, x.data_ptr(), 16, w.data_ptr(), 16, t.data_ptr(), None, 1.0, 0)
    out = torch.empty(20, device="cuda")
    p = lambda q: ctypes.c_void_p(q.data_ptr())
    small = torch.empty(512, dtype=torch.uint8, device="cuda")
    assert pkg.lib.ivfr_softmax_loss(ctypes.byref(a), p(out), p(out), p(small), 16, None) == pkg.binding.ERR_INVALID_ARG
    assert b"are needed" in pkg.lib.ivfr_last_error()
