"""Root-mean-square norm, its 8-bit output and its backward pass against their formulas in 64 bits.

Tolerances, from the arithmetic (u: half a unit in the last place of the output's type, e = 2^-24): a float32 sum of d terms
whose longest chain of additions is d/256 + 16 is off by at most A = (d/256 + 16) e of the sum of the magnitudes, rstd by half of
that and a few e.  The sums over rows have chains of at most rows/256 + 300.  An 8-bit number is off by 2^-4 of its value, or by
2^-10 where it is below 2^-6.
"""

import math

import pytest

import torch

from lm_common import DEV, EPS, LEAST, TYPES, UNIT, apart, gen, within

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn
SHAPES = [(1, 1), (2, 2), (5, 7), (1, 4096), (3, 63), (64, 64), (17, 257), (33, 1000), (7, 1111), (300, 128), (9, 2047), (6, 2048),
          (4, 2049), (5, 4097), (3, 8192), (3, 8200), (2, 16384), (2, 16385), (2, 40001), (1000, 96), (2051, 260)]


def _inputs(rows, d, type, seed, weights):
    g = gen(seed)
    spread = 0.5 + torch.rand((rows, 1), generator=g, device=DEV)
    x, r, dy, ds = (torch.randn((rows, d), generator=g, device=DEV).mul(spread).to(TYPES[type]) for _ in range(4))
    w = None
    if weights:
        w = (1.0 + 0.2 * torch.randn((d,), generator=g, device=DEV)).to(TYPES[type] if weights == "own" else torch.float32)
    return x, r, w, (dy * 0.1).to(x.dtype), (ds * 0.1).to(x.dtype)


def _chain(n, more=16):
    return (math.ceil(n / 256) + more) * EPS


def _check_forward(got, x, r, w, eps, type):
    y, total, scale, rstd = got
    h = x
    if r is None:
        assert total is None
    else:
        h = (x.float() + r.float()).to(x.dtype)
        assert torch.equal(total, h)
    h = h.double()
    err = _chain(x.shape[1]) + 8 * EPS
    rs = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    within(rstd[:, None], rs, err * rs, "rstd")
    want = h * rs * (1.0 if w is None else w.double())
    if y.dtype != E4M3:
        assert scale is None and y.dtype == x.dtype
        within(y, want, UNIT[type] * want.abs() + LEAST[type] + want.abs() * err * (1 + UNIT[type]), "y")
        return
    s = want.abs().amax(1, keepdim=True) / 448
    within(scale[:, None], s, (err + 4 * EPS) * s + 2.0 ** -149, "scale")
    q = want / s
    moved = 2 * err + 8 * EPS
    within(y, q, q.abs() * (2.0 ** -4 * (1 + moved) + moved) + 2.0 ** -10, "q")


def _grad(dy, ds, h, w, rstd):
    """dx, dweight by the formula in 64 bits."""
    rs = rstd.double()[:, None]
    n, g = h.double() * rs, dy.double() * (1.0 if w is None else w.double())
    dx = rs * (g - n * (g * n).mean(1, keepdim=True))
    return dx if ds is None else dx + ds.double(), (dy.double() * n).sum(0)


def _dx_tolerance(dy, ds, h, w, rstd, want, type):
    rs = rstd.double()[:, None]
    n, g = h.double() * rs, dy.double() * (1.0 if w is None else w.double())
    a = (g * n).mean(1, keepdim=True)
    ea = (_chain(h.shape[1]) + 4 * EPS) * (g * n).abs().mean(1, keepdim=True)
    inner = rs * (n.abs() * ea + 6 * EPS * (g.abs() + (n * a).abs())) + 2 * EPS * want.abs()
    return UNIT[type] * want.abs() + LEAST[type] + inner * (1 + UNIT[type]) + (0.0 if ds is None else 2 * EPS * ds.double().abs())


def _check_backward(got, dy, ds, h, w, rstd, type):
    dx, dw = got
    want, want_w = _grad(dy, ds, h, w, rstd)
    within(dx, want, _dx_tolerance(dy, ds, h, w, rstd, want, type), "dx")
    rows = h.shape[0]
    n = h.double() * rstd.double()[:, None]
    within(dw, want_w, (_chain(rows, 300) + 4 * EPS) * (dy.double() * n).abs().sum(0), "dweight")


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("rows,d", SHAPES)
def test_forward_and_backward(rows, d, type):
    import paper_1704_07355_amd as Q
    for weights in ("f32", "own", None):
        x, r, w, dy, ds = _inputs(rows, d, type, rows * 31 + d, weights)
        for res in (None, r):
            for out_type in (None, E4M3):
                got = Q.qadc_rms_norm(x, w, res, 1e-5, out_type)
                _check_forward(got, x, res, w, 1e-5, type)
            h, rstd = x if res is None else got[1], got[3]
            for more in (None, ds):
                _check_backward(Q.qadc_rms_norm_backward(dy, h, w, rstd, more), dy, more, h, w, rstd, type)


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("rows,d,ld,shift", [(9, 100, 101, 1), (300, 257, 300, 3), (5, 4096, 5001, 7), (1, 33, 40, 5), (40, 8, 8, 1),
                                             (3, 17001, 17003, 3)])
def test_rows_apart_and_unaligned(rows, d, ld, shift, type):
    import paper_1704_07355_amd as Q
    x, r, w, dy, ds = _inputs(rows, d, type, ld, "f32")
    xs, rs, dys, dss = apart(x, ld, shift), apart(r, ld + 3, shift), apart(dy, ld + 2, shift + 1), apart(ds, ld + 1, shift + 2)
    room = apart(x, ld + 5, shift)
    for out_type in (None, E4M3):
        a, c = Q.qadc_rms_norm(x, w, r, 1e-5, out_type), Q.qadc_rms_norm(xs, w, rs, 1e-5, out_type, sum_out=room)
        assert all(p is q is None or torch.equal(p.float(), q.float()) for p, q in zip(a, c))
    between = torch.as_strided(room, (rows - 1, 5), (ld + 5, 1), room.storage_offset() + d) if rows > 1 else room[:0]
    assert torch.isnan(between.float()).all()  # what lies between the rows is left as it was
    a, c = Q.qadc_rms_norm_backward(dy, a[1], w, a[3], ds), Q.qadc_rms_norm_backward(dys, room, w, c[3], dss)
    assert all(torch.equal(p, q) for p, q in zip(a, c))


@pytest.mark.parametrize("type", list(TYPES))
def test_in_place(type):
    import paper_1704_07355_amd as Q
    for rows, d in ((37, 1000), (4, 20001), (700, 130), (1500, 4096)):
        x, r, w, dy, ds = _inputs(rows, d, type, 5, "f32")
        y, total, _, rstd = Q.qadc_rms_norm(x, w, r)
        for sum_at in ("x", "r", None):
            for y_at in ("x", "r", None):
                if sum_at is not None and sum_at == y_at:
                    continue
                x2, r2 = x.clone(), r.clone()
                at = {"x": x2, "r": r2, None: None}
                got = Q.qadc_rms_norm(x2, w, r2, sum_out=at[sum_at], out=at[y_at])
                assert torch.equal(got[0], y) and torch.equal(got[1], total) and torch.equal(got[3], rstd)
        want = Q.qadc_rms_norm_backward(dy, total, w, rstd, ds)
        for target in ("dy", "h", "ds"):
            at = {"dy": dy.clone(), "h": total.clone(), "ds": ds.clone()}
            got = Q.qadc_rms_norm_backward(at["dy"], at["h"], w, rstd, at["ds"], out=at[target])
            assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_zeros_tiny_large_and_broken_rows():
    import paper_1704_07355_amd as Q
    for d in (500, 20000):
        x = torch.ones((7, d), device=DEV)
        x[0] = 0.0
        x[1, 3] = math.inf
        x[2, d - 1] = math.nan
        x[3] = 1e-30     # far below eps
        x[4] = 1e15
        x[5, :] = 0.0
        x[5, d // 2] = -3.0
        y, _, scale, rstd = Q.qadc_rms_norm(x, None, None, 1e-5, E4M3)
        y = y.float()
        assert (y[0] == 0).all() and scale[0] == 0
        assert torch.isnan(y[1:3]).all() and torch.isnan(scale[1:3]).all()
        assert (y[3] == 448).all() and abs(scale[3].item() * 448 / (1e-30 / math.sqrt(1e-5)) - 1) < 1e-5
        assert (y[4] == 448).all() and abs(scale[4].item() * 448 - 1) < 1e-5
        assert y[5, d // 2] == -448 and (y[5] != 0).sum() == 1
        # the smallest values: below 448 / 2^126 the range is not used up, the values still come back
        tiny = torch.full((2, d), 2.0 ** -130, device=DEV)
        q, _, s, _ = Q.qadc_rms_norm(tiny, None, None, 1.0, E4M3)
        assert (q.double() * s.double()[:, None] - 2.0 ** -130).abs().max() <= 2.0 ** -10 * 2.0 ** -126
        # eps = 0: a row of zeros has no direction
        z, _, _, rs = Q.qadc_rms_norm(torch.zeros((1, d), device=DEV), eps=0.0)
        assert torch.isinf(rs).all() and torch.isnan(z).all()
        # beyond what float32 squares hold
        big, _, _, _ = Q.qadc_rms_norm(torch.full((1, d), 1e25, device=DEV))
        assert (big == 0).all()


@pytest.mark.parametrize("type", list(TYPES))
def test_rows_with_infinities(type):
    """In 8 bits the row is NaN; of the rows' type its infinite elements are, and the others vanish beside them.  Its neighbours stay."""
    import paper_1704_07355_amd as Q
    for d in (64, 500, 20000):
        x, r, w, dy, _ = _inputs(5, d, type, d, "f32")
        x[1, 3], x[3, d - 1], r[3, 7] = math.inf, -math.inf, math.nan
        for eps in (1e-5, 0.0):
            y, total, _, rstd = Q.qadc_rms_norm(x, w, r, eps)
            assert torch.isnan(y[1, 3]) and torch.isnan(y[1]).sum() == 1 and (y[1].nan_to_num() == 0).all() and rstd[1] == 0
            assert torch.isnan(y[3]).all() and torch.isnan(rstd[3])
            q, _, scale, _ = Q.qadc_rms_norm(x, w, r, eps, E4M3)
            assert torch.isnan(q[1].float()).all() and torch.isnan(q[3].float()).all() and torch.isnan(scale[[1, 3]]).all()
            dx, _ = Q.qadc_rms_norm_backward(dy, total, w, rstd)
            assert torch.isnan(dx[[1, 3]]).all()
            rest = [0, 2, 4]
            alone = Q.qadc_rms_norm(x[rest], w, r[rest], eps)
            assert torch.equal(y[rest], alone[0]) and torch.equal(rstd[rest], alone[3]) and torch.equal(
                dx[rest], Q.qadc_rms_norm_backward(dy[rest], alone[1], w, alone[3])[0])


def _equal(a, b):
    return all(p is q is None or torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("eps", [0.0, 2.0 ** -146, 2.0 ** -116])
def test_rows_so_small_that_their_squares_are_not_float32(eps, type):
    """Rows without an eps that outweighs them, small ones beside ordinary ones in a workgroup: each as if it was alone."""
    import paper_1704_07355_amd as Q
    sizes = [1.0, 1e-4, 2.0 ** -12] if type == "f16" else [1.0, 1e-15, 1e-19, 1e-21, 1e-23, 1e-30, 1e-36]
    for d in (1, 7, 100, 130, 300, 1000, 1500, 4096, 5003, 12000, 16385):
        g = torch.Generator().manual_seed(d)
        size = torch.tensor([sizes[i % len(sizes)] for i in range(23)], dtype=torch.float64)[:, None]
        x, r = ((0.5 + torch.rand((23, d), generator=g, dtype=torch.float64)) * size for _ in range(2))
        x, r = x.to(TYPES[type]).to(DEV), (0.3 * r).to(TYPES[type]).to(DEV)
        w = (1.0 + 0.2 * torch.randn((d,), generator=g)).to(DEV)
        dy, ds = (0.1 * torch.randn((23, d), generator=g).to(TYPES[type]).to(DEV) for _ in range(2))
        for weight in (w, None):
            for res in (None, r):
                for out_type in (None, E4M3):
                    got = Q.qadc_rms_norm(x, weight, res, eps, out_type)
                    _check_forward(got, x, res, weight, eps, type)
                h, rstd = x if res is None else got[1], got[3]
                _check_backward(Q.qadc_rms_norm_backward(dy, h, weight, rstd, ds), dy, ds, h, weight, rstd, type)
        one = Q.qadc_rms_norm(x[6:7], w, r[6:7], eps)
        whole = Q.qadc_rms_norm(x, w, r, eps)
        assert _equal(one, [None if t is None else t[6:7] for t in whole])
        # in place, and rows apart
        x2, r2 = apart(x, d + 3, 1), r.clone()
        assert _equal(Q.qadc_rms_norm(x2, w, r2, eps, sum_out=x2, out=r2), whole)


@pytest.mark.parametrize("type", ["f32", "bf16"])
def test_rows_beyond_the_smallest_reciprocal(type):
    """Without an eps, rows of a root mean square below 2^-128 have a y, but no float32 holds their rstd."""
    import paper_1704_07355_amd as Q
    least = 2.0 ** -149 if type == "f32" else 2.0 ** -133
    for d in (3, 200, 4097, 20000):
        steps = torch.randint(1, 9, (4, d), generator=torch.Generator().manual_seed(d))
        x = (steps.double() * least).to(TYPES[type]).to(DEV)
        want = steps.double().to(DEV)
        want = want / torch.sqrt((want * want).mean(1, keepdim=True))
        err = _chain(d) + 8 * EPS
        y, _, _, rstd = Q.qadc_rms_norm(x, eps=0.0)
        within(y, want, UNIT[type] * want + want * err * (1 + UNIT[type]), "y")
        assert torch.isinf(rstd).all()
        q, _, scale, _ = Q.qadc_rms_norm(x, eps=0.0, out_type=E4M3)
        s = want.amax(1, keepdim=True) / 448
        within(scale[:, None], s, (err + 4 * EPS) * s, "scale")
        moved = 2 * err + 8 * EPS
        within(q, want / s, want / s * (2.0 ** -4 * (1 + moved) + moved) + 2.0 ** -10, "q")
        # an eps of their size
        for eps in (2.0 ** -149, 2.0 ** -140):
            y, _, _, rstd = Q.qadc_rms_norm(x, eps=eps)
            rs = 1 / torch.sqrt((x.double() * x.double()).mean(1, keepdim=True) + eps)
            within(rstd[:, None], rs, err * rs, "rstd")
            within(y, x.double() * rs, UNIT[type] * x.double() * rs + LEAST[type] + x.double() * rs * err * (1 + UNIT[type]), "y")
    zero = torch.zeros((2, 300), dtype=TYPES[type], device=DEV)
    y, _, _, rstd = Q.qadc_rms_norm(zero, eps=2.0 ** -149)
    assert (y == 0).all() and torch.equal(rstd, torch.full_like(rstd, 2.0 ** 74.5))
    q, _, scale, _ = Q.qadc_rms_norm(zero, eps=0.0, out_type=E4M3)
    assert torch.isnan(q.float()).all() and torch.isnan(scale).all()


def test_the_gradient_of_a_very_long_weight(memory_back):
    """More columns than the threads of a launch in one direction reach, sixteen a column, would be."""
    import paper_1704_07355_amd as Q
    rows, d = 2, (1 << 28) + 37
    h, dy = (torch.randn((rows, d), generator=gen(s), device=DEV, dtype=torch.bfloat16) for s in (1, 2))
    rstd = torch.tensor([0.7, 1.9], device=DEV)
    none, dw = Q.qadc_rms_norm_backward(dy, h, None, rstd, need_dx=False)
    for c in range(0, d, 1 << 26):
        n = h[:, c:c + (1 << 26)].double() * rstd.double()[:, None]
        g = dy[:, c:c + (1 << 26)].double()
        within(dw[c:c + (1 << 26)], (g * n).sum(0), (_chain(rows, 300) + 4 * EPS) * (g * n).abs().sum(0), "dweight")


def test_gradient_against_differences():
    """Central differences of sum(dy y) + sum(dsum h) in 64 bits, along random directions of x and of the weight."""
    import paper_1704_07355_amd as Q
    for rows, d in ((3, 50), (2, 1000)):
        x, _, w, dy, ds = _inputs(rows, d, "f32", 9, "f32")
        rstd = Q.qadc_rms_norm(x, w)[3]
        dx, dw = Q.qadc_rms_norm_backward(dy, x, w, rstd, ds)

        def value(x, w):
            return (dy.double() * (x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-5) * w)).sum() + (ds.double() * x).sum()

        g = gen(4)
        for _ in range(4):
            u = torch.randn((rows, d), generator=g, device=DEV).double()
            v = torch.randn((d,), generator=g, device=DEV).double()
            t = 1e-4
            slope = (value(x.double() + t * u, w.double() + t * v) - value(x.double() - t * u, w.double() - t * v)) / (2 * t)
            want, want_w = _grad(dy, ds, x, w, rstd)
            # float32 errors of the gradients, rstd's own (A + 8 e) in both, and t^2 of a third derivative of the size of the values
            tol = (_dx_tolerance(dy, ds, x, w, rstd, want, "f32") * u.abs()).sum() + 400 * EPS * (want_w.abs() * v.abs()).sum() \
                + (_chain(d) + 8 * EPS) * 4 * ((want.abs() * u.abs()).sum() + (want_w.abs() * v.abs()).sum()) \
                + 10 * t * t * (dy.double().abs() * (u.abs() + v.abs()) ** 3).sum()
            assert abs(((dx.double() * u).sum() + (dw.double() * v).sum() - slope).item()) <= tol.item()


def test_equal_calls_give_equal_bits_and_a_workspace_serves_fewer_rows():
    import paper_1704_07355_amd as Q
    x, _, w, dy, ds = _inputs(3000, 640, "bf16", 3, "f32")
    rstd = Q.qadc_rms_norm(x, w)[3]
    ws = torch.empty(Q.qadc_rms_norm_workspace_bytes(3000, 640), dtype=torch.uint8, device=DEV)
    a = Q.qadc_rms_norm_backward(dy, x, w, rstd, ds, workspace=ws)
    ws.fill_(255)
    b = Q.qadc_rms_norm_backward(dy, x, w, rstd, ds, workspace=ws)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    for rows in (1, 2, 511, 512, 513, 2999):
        Q.qadc_rms_norm_backward(dy[:rows], x[:rows], w, rstd[:rows], workspace=ws)
    for d in (64, 1024, 4096, 5000, 16384, 20000):
        most = Q.qadc_rms_norm_workspace_bytes(4097, d)
        assert all(Q.qadc_rms_norm_workspace_bytes(r, d) <= most for r in (1, 2, 16, 255, 256, 257, 511, 512, 513, 1025, 4096))


def test_parts_of_the_gradient_and_no_rows():
    import paper_1704_07355_amd as Q
    x, _, w, dy, _ = _inputs(40, 300, "f16", 3, "own")
    rstd = Q.qadc_rms_norm(x, w)[3]
    dx, dw = Q.qadc_rms_norm_backward(dy, x, w, rstd)
    a, none = Q.qadc_rms_norm_backward(dy, x, w, rstd, need_weight=False)
    assert none is None and torch.equal(a, dx)
    none, b = Q.qadc_rms_norm_backward(dy, x, w, rstd, need_dx=False)
    assert none is None and torch.equal(b, dw)
    y, total, scale, rs = Q.qadc_rms_norm(x[:0], w, x[:0], 1e-5, E4M3)
    assert y.shape == (0, 300) and total.shape == (0, 300) and scale.numel() == rs.numel() == 0
    dx, dw = Q.qadc_rms_norm_backward(dy[:0], x[:0], w, rstd[:0])
    assert dx.shape == (0, 300) and (dw == 0).all()


def test_wrong_tensors_are_refused():
    import paper_1704_07355_amd as Q
    x, r, w, dy, ds = _inputs(4, 64, "f16", 3, "f32")
    rstd = Q.qadc_rms_norm(x, w)[3]
    for call in (lambda: Q.qadc_rms_norm(x, w.double()), lambda: Q.qadc_rms_norm(x, w[:63]), lambda: Q.qadc_rms_norm(x, w, r[:3]),
                 lambda: Q.qadc_rms_norm(x, w, r.float()), lambda: Q.qadc_rms_norm(x, w, r, out_type=torch.float32),
                 lambda: Q.qadc_rms_norm(x, w, sum_out=r), lambda: Q.qadc_rms_norm(x, w, out_type=E4M3, out=torch.empty_like(x)),
                 lambda: Q.qadc_rms_norm(x.t(), w), lambda: Q.qadc_rms_norm(x.cpu(), w),
                 lambda: Q.qadc_rms_norm_backward(dy[:3], x, w, rstd), lambda: Q.qadc_rms_norm_backward(dy, x, w, rstd, ds[:3]),
                 lambda: Q.qadc_rms_norm_backward(dy, x, w, rstd[:3]), lambda: Q.qadc_rms_norm_backward(dy.float(), x, w, rstd)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(Q.QadcError):
        Q.qadc_rms_norm(x, w, r, sum_out=x, out=x)
    with pytest.raises(Q.QadcError):
        Q.qadc_rms_norm_backward(dy, x, w, rstd, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
