"""Layer norm and its backward pass against their formulas in 64 bits.

Tolerances, from the arithmetic (u: half a unit in the last place of the output's type, e = 2^-24): a float32 sum of d terms
whose longest chain of additions is d/256 + 16 is off by at most A = (d/256 + 16) e of the sum of the magnitudes.  The mean is
then off by at most A mean|x|, the variance by 2A relative and the mean's error squared, rstd by half of that and a few e.
The sums over rows have chains of at most rows/256 + 300.
"""

import math

import pytest

import torch

from lm_common import DEV, EPS, LEAST, TYPES, UNIT, apart, gen, within

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (2, 2), (5, 7), (1, 4096), (3, 63), (64, 64), (17, 257), (33, 1000), (7, 1111), (300, 128), (9, 2047), (6, 2048),
          (4, 2049), (5, 4097), (3, 8192), (2, 16384), (2, 16385), (2, 40001), (1000, 96), (2051, 260)]


def _inputs(rows, d, type, seed, weights):
    g = gen(seed)
    x = torch.randn((rows, d), generator=g, device=DEV) * (0.5 + torch.rand((rows, 1), generator=g, device=DEV))
    x = (x + 2.0 * torch.randn((rows, 1), generator=g, device=DEV)).to(TYPES[type])
    w = b = None
    if weights:
        t = TYPES[type] if weights == "own" else torch.float32
        w = (1.0 + 0.2 * torch.randn((d,), generator=g, device=DEV)).to(t)
        b = (0.3 * torch.randn((d,), generator=g, device=DEV)).to(t)
    return x, w, b, (0.1 * torch.randn((rows, d), generator=g, device=DEV)).to(TYPES[type])


def _check_forward(got, x, w, b, eps, type):
    y, mean, rstd = got
    x64 = x.double()
    d = x.shape[1]
    A = (math.ceil(d / 256) + 16) * EPS
    mu = x64.mean(1, keepdim=True)
    c = x64 - mu
    var = (c * c).mean(1, keepdim=True)
    rs = 1 / torch.sqrt(var + eps)
    w64 = 1.0 if w is None else w.double()
    b64 = 0.0 if b is None else b.double()
    emean = A * x64.abs().mean(1, keepdim=True) + EPS * mu.abs()
    ers = (2 * A + 8 * EPS) + (emean * rs) ** 2 + emean * rs * 2 * A
    h = c * rs
    want = h * w64 + b64
    within(mean[:, None], mu, emean, "mean")
    within(rstd[:, None], rs, ers * rs, "rstd")
    tol = UNIT[type] * want.abs() + LEAST[type] + (h.abs() * ers + rs * emean) * abs(w64) * (1 + UNIT[type]) \
        + 4 * EPS * ((h * w64).abs() + abs(b64) + torch.zeros_like(h))
    within(y, want, tol, "y")


def _check_backward(got, dy, x, w, mean, rstd, type):
    dx, dw, db = got
    rows, d = x.shape
    A = (math.ceil(d / 256) + 16) * EPS
    B = (math.ceil(rows / 256) + 300) * EPS
    dy64, mu, rs = dy.double(), mean.double()[:, None], rstd.double()[:, None]
    h = (x.double() - mu) * rs
    eh = 3 * EPS * (h.abs() + mu.abs() * rs)
    g = dy64 * (1.0 if w is None else w.double())
    a, b = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    want = rs * (g - a - h * b)
    ea = (A + 2 * EPS) * g.abs().mean(1, keepdim=True)
    eb = (A + 4 * EPS) * (g * h).abs().mean(1, keepdim=True) + (g.abs() * eh).mean(1, keepdim=True)
    inner = ea + h.abs() * eb + eh * b.abs() + 6 * EPS * (g.abs() + a.abs() + (h * b).abs())
    within(dx, want, UNIT[type] * want.abs() + LEAST[type] + rs * inner * (1 + UNIT[type]), "dx")
    within(dw, (dy64 * h).sum(0), (B + 4 * EPS) * (dy64 * h).abs().sum(0) + (dy64.abs() * eh).sum(0), "dweight")
    within(db, dy64.sum(0), B * dy64.abs().sum(0), "dbias")


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("rows,d", SHAPES)
def test_forward_and_backward(rows, d, type):
    import paper_1704_07355_amd as Q
    for weights in ("f32", "own", None):
        x, w, b, dy = _inputs(rows, d, type, rows * 31 + d, weights)
        got = Q.qadc_layer_norm(x, w, b, 1e-5)
        _check_forward(got, x, w, b, 1e-5, type)
        _, mean, rstd = got
        _check_backward(Q.qadc_layer_norm_backward(dy, x, w, mean, rstd), dy, x, w, mean, rstd, type)


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("rows,d,ld,shift", [(9, 100, 101, 1), (300, 257, 300, 3), (5, 4096, 5001, 7), (1, 33, 40, 5), (40, 8, 8, 1)])
def test_rows_apart_and_unaligned(rows, d, ld, shift, type):
    import paper_1704_07355_amd as Q
    x, w, b, dy = _inputs(rows, d, type, ld, "f32")
    xs, dys = apart(x, ld, shift), apart(dy, ld + 2, shift + 1)
    a, c = Q.qadc_layer_norm(x, w, b), Q.qadc_layer_norm(xs, w, b)
    assert all(torch.equal(p, q) for p, q in zip(a, c))
    a = Q.qadc_layer_norm_backward(dy, x, w, a[1], a[2])
    c = Q.qadc_layer_norm_backward(dys, xs, w, c[1], c[2])
    assert all(torch.equal(p, q) for p, q in zip(a, c))


@pytest.mark.parametrize("type", list(TYPES))
def test_in_place(type):
    import paper_1704_07355_amd as Q
    for rows, d in ((37, 1000), (4, 20001), (700, 130)):
        x, w, b, dy = _inputs(rows, d, type, 5, "f32")
        y, mean, rstd = Q.qadc_layer_norm(x, w, b)
        want = Q.qadc_layer_norm_backward(dy, x, w, mean, rstd)
        for target in ("dy", "x"):
            x2, dy2 = x.clone(), dy.clone()
            got = Q.qadc_layer_norm_backward(dy2, x2, w, mean, rstd, out=dy2 if target == "dy" else x2)
            assert all(torch.equal(p, q) for p, q in zip(got, want))
        x2 = x.clone()
        Q.qadc_layer_norm(x2, w, b, out=x2)
        assert torch.equal(x2, y)


def test_constant_rows_large_offsets_and_eps():
    import paper_1704_07355_amd as Q
    # a row of equal values has no variance: y is the bias, rstd 1 / sqrt(eps)
    x = torch.full((3, 500), 7.0, device=DEV)
    b = torch.randn((500,), generator=gen(1), device=DEV)
    y, mean, rstd = Q.qadc_layer_norm(x, None, b, 1e-4)
    assert torch.equal(y, b.expand(3, 500)) and torch.equal(mean, torch.full((3,), 7.0, device=DEV))
    within(rstd, torch.full((3,), 100.0, device=DEV, dtype=torch.float64), 1e-4)
    # eps = 0 divides by zero there: NaN, and nothing else is touched
    y, _, rstd = Q.qadc_layer_norm(torch.cat((x, torch.randn((1, 500), generator=gen(2), device=DEV))), None, None, 0.0)
    assert torch.isnan(y[:3]).all() and torch.isinf(rstd[:3]).all() and torch.isfinite(y[3]).all()
    # a spread of 1 around 4096: a difference of squares would lose it
    x = 4096.0 + torch.randn((50, 777), generator=gen(3), device=DEV)
    _check_forward(Q.qadc_layer_norm(x), x, None, None, 1e-5, "f32")


def test_rows_that_are_not_finite_stay_alone():
    import paper_1704_07355_amd as Q
    x, w, b, dy = _inputs(64, 300, "bf16", 9, "f32")
    clean = Q.qadc_layer_norm(x, w, b)
    x2 = x.clone()
    x2[5, 17], x2[40, 0], x2[41, 299] = math.inf, math.nan, -math.inf
    y, mean, rstd = Q.qadc_layer_norm(x2, w, b)
    bad = torch.zeros((64,), dtype=torch.bool, device=DEV)
    bad[[5, 40, 41]] = True
    assert torch.isnan(y[bad]).all() and torch.equal(y[~bad], clean[0][~bad])
    dx, dw, _ = Q.qadc_layer_norm_backward(dy, x2, w, mean, rstd)
    assert torch.isnan(dx[bad]).all() and torch.isfinite(dx[~bad]).all() and torch.isnan(dw).all()


@pytest.mark.parametrize("rows,d", [(40, 300), (3, 2000)])
def test_gradient_by_differences(rows, d):
    """d/dh of sum(c y) along a direction, by central differences with h = 2^-8: off by h^2 times the third derivative (of order
    one per unit of x) and by the rounding of y, 2^-22 sqrt(rows d) / h."""
    import paper_1704_07355_amd as Q
    g = gen(rows)
    x, w, b, c = _inputs(rows, d, "f32", 77, "f32")
    _, mean, rstd = Q.qadc_layer_norm(x, w, b)
    dx, dw, db = Q.qadc_layer_norm_backward(c, x, w, mean, rstd)
    loss = lambda x, w, b: (Q.qadc_layer_norm(x, w, b)[0].double() * c.double()).sum().item()
    h = 2.0 ** -8
    for grad, at in ((dx, 0), (dw, 1), (db, 2)):
        # along the gradient itself, so that the derivative is not a difference of large numbers
        e = grad / grad.abs().max()
        hi, lo = [x, w, b], [x, w, b]
        hi[at], lo[at] = hi[at] + h * e, lo[at] - h * e
        want = (loss(*hi) - loss(*lo)) / (2 * h)
        got = (grad.double() * e.double()).sum().item()
        size = c.double().norm().item()
        assert abs(got - want) <= 20 * h * h * abs(got) + 2.0 ** -22 * size * 4 / h, (at, got, want)


def test_no_rows_and_optional_outputs():
    import paper_1704_07355_amd as Q
    x, w, b, dy = _inputs(20, 333, "f16", 3, "own")
    y, mean, rstd = Q.qadc_layer_norm(x[:0], w, b)
    assert y.shape == (0, 333) and mean.shape == (0,)
    dx, dw, db = Q.qadc_layer_norm_backward(dy[:0], x[:0], w, mean, rstd)
    assert dx.shape == (0, 333) and not dw.any() and not db.any() and dw.shape == (333,)
    _, mean, rstd = Q.qadc_layer_norm(x, w, b)
    all3 = Q.qadc_layer_norm_backward(dy, x, w, mean, rstd)
    only = Q.qadc_layer_norm_backward(dy, x, w, mean, rstd, need_weights=False)
    assert torch.equal(only[0], all3[0]) and only[1] is None
    only = Q.qadc_layer_norm_backward(dy, x, w, mean, rstd, need_dx=False)
    assert only[0] is None and torch.equal(only[1], all3[1]) and torch.equal(only[2], all3[2])


def test_equal_calls_give_equal_bits_and_streams():
    import paper_1704_07355_amd as Q
    x, w, b, dy = _inputs(5000, 520, "bf16", 8, "f32")
    _, mean, rstd = Q.qadc_layer_norm(x, w, b)
    ws = torch.empty((Q.qadc_layer_norm_workspace_bytes(5000, 520),), dtype=torch.uint8, device=DEV)
    first = Q.qadc_layer_norm_backward(dy, x, w, mean, rstd, workspace=ws)
    ws.fill_(0xFF)  # the workspace need not be cleared
    again = Q.qadc_layer_norm_backward(dy, x, w, mean, rstd, workspace=ws)
    assert all(torch.equal(p, q) for p, q in zip(first, again))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        other = Q.qadc_layer_norm_backward(dy, x, w, mean, rstd, workspace=ws)
    s.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(first, other))


def test_offsets_beyond_32_bits():
    import paper_1704_07355_amd as Q
    x, w, b, dy = _inputs(3, 1000, "bf16", 4, "f32")
    ld = 1_500_000_000
    buf = torch.empty((2 * ld + 1000,), dtype=torch.bfloat16, device=DEV)
    far = torch.as_strided(buf, (3, 1000), (ld, 1))
    far.copy_(x)
    want = Q.qadc_layer_norm(x, w, b)
    got = Q.qadc_layer_norm(far, w, b)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    a = Q.qadc_layer_norm_backward(dy, x, w, want[1], want[2])
    c = Q.qadc_layer_norm_backward(dy, far, w, want[1], want[2])
    assert all(torch.equal(p, q) for p, q in zip(a, c))


def test_refusals_of_the_binding():
    import paper_1704_07355_amd as Q
    x, w, b, dy = _inputs(6, 40, "f16", 1, "own")
    _, mean, rstd = Q.qadc_layer_norm(x, w, b)
    for bad in (lambda: Q.qadc_layer_norm(x.double()), lambda: Q.qadc_layer_norm(x.t()), lambda: Q.qadc_layer_norm(x.cpu()),
                lambda: Q.qadc_layer_norm(x, w[:39]), lambda: Q.qadc_layer_norm(x, w, b.float()),
                lambda: Q.qadc_layer_norm(x, w.bfloat16()), lambda: Q.qadc_layer_norm(x[:1].expand(6, 40)),
                lambda: Q.qadc_layer_norm(x, out=torch.empty((6, 41), dtype=x.dtype, device=DEV)),
                lambda: Q.qadc_layer_norm_backward(dy[:5], x, w, mean, rstd),
                lambda: Q.qadc_layer_norm_backward(dy.float(), x, w, mean, rstd),
                lambda: Q.qadc_layer_norm_backward(dy, x, w, mean[:5], rstd)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(Q.QadcError):
        Q.qadc_layer_norm(x, w, b, -1.0)
    with pytest.raises(Q.QadcError) as e:
        Q.qadc_layer_norm_backward(dy, x, w, mean, rstd, workspace=torch.empty((16,), dtype=torch.uint8, device=DEV))
    assert e.value.code == Q.QADC_ENOMEM


@pytest.mark.parametrize("rows,d", [(513, 4096), (2100, 900), (257, 8000), (8200, 20000)])
def test_a_workspace_for_a_batch_serves_its_smaller_batches(rows, d):
    import paper_1704_07355_amd as Q
    ws = torch.empty((Q.qadc_layer_norm_workspace_bytes(rows, d),), dtype=torch.uint8, device=DEV)
    x, w, b, dy = _inputs(rows, d, "bf16", 41, "f32")
    _, mean, rstd = Q.qadc_layer_norm(x, w, b)
    for n in (rows, rows - 1, rows // 2 + 200, 256, 3):
        if n > rows:
            continue
        part = dy[:n], x[:n], w, mean[:n], rstd[:n]
        got, want = Q.qadc_layer_norm_backward(*part, workspace=ws), Q.qadc_layer_norm_backward(*part)
        assert all(torch.equal(p, q) for p, q in zip(got, want)), n


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("rows,d", [(3000, 100), (2051, 260), (700, 1111), (1100, 4096), (300, 8000), (270, 12000), (40, 20001)])
def test_rows_alone_give_the_bits_they_give_among_others(rows, d, type):
    import paper_1704_07355_amd as Q
    x, w, b, dy = _inputs(rows, d, type, 42, "f32")
    y, mean, rstd = Q.qadc_layer_norm(x, w, b)
    dx, _, _ = Q.qadc_layer_norm_backward(dy, x, w, mean, rstd)
    for r in (0, 1, rows // 2, rows - 1):
        one = slice(r, r + 1)
        assert all(torch.equal(p[0], q[r]) for p, q in zip(Q.qadc_layer_norm(x[one], w, b), (y, mean, rstd)))
        assert torch.equal(Q.qadc_layer_norm_backward(dy[one], x[one], w, mean[one], rstd[one])[0][0], dx[r])
