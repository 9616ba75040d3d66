"""Log probabilities of given tokens, entropy, alternatives and their gradient against the formulas in 64 bits.

Tolerances, with e = 2^-24: the exponent x - m of a token is off by at most ex = 6 e (|x| + |m| + |x - m|) (the scaled logit, the
difference, a factor of log 2), so its exponential by ex + 4 e relative, and a sum over V by (V / 256 + 40) e more.  The
alternatives' tokens are whole numbers and have to be equal.
"""

import math

import pytest

import torch

from lm_common import DEV, EPS, LEAST, TYPES, UNIT, apart, gen, within

pytestmark = pytest.mark.gpu


def make(rows, V, type, seed, masked=0.0, spread=3.0):
    g = gen(seed)
    x = spread * torch.randn((rows, V), generator=g, device=DEV)
    at = torch.randint(0, V, (rows, 5), generator=g, device=DEV)
    x.scatter_add_(1, at, 6.0 * torch.rand((rows, 5), generator=g, device=DEV))
    if masked:
        x.masked_fill_(torch.rand((rows, V), generator=g, device=DEV) < masked, -math.inf)
    return x.to(TYPES[type])


def make_tokens(rows, V, T, seed):
    g = gen(seed)
    t = torch.randint(0, V, (rows, T), generator=g, device=DEV, dtype=torch.int32)
    if T > 3:
        t[:, 1] = t[:, 0]            # given twice
        t[::2, 2] = -1               # unused slots
        t[1::2, 3] = V
    return t


def reference(logits, scale):
    """x, m, p and the bound q of p's relative error, in 64 bits; rows with nothing left have p = 0."""
    x = logits.double() * scale
    V = x.shape[1]
    m = x.max(1, keepdim=True).values
    some = torch.isfinite(m)
    d = torch.where(some & (x > -math.inf), x - torch.where(some, m, 0.0), -math.inf)
    e = torch.exp(d)
    s = e.sum(1, keepdim=True)
    p = torch.where(some, e / s, 0.0)
    dz = torch.where(e > 0, d, 0.0)
    xz = torch.where(e > 0, x, 0.0)
    ex = torch.where(e > 0, 6 * EPS * (xz.abs() + m.abs().nan_to_num(0, 0, 0) + dz.abs()), 0.0)
    q = ex + (V / 256 + 44) * EPS
    return x, m, s, p, dz, ex, q


def check(got, logits, tokens, k, scale):
    """Rows of finite and masked logits, at least one finite."""
    logp, lse, H, top, top_logp = got
    rows, V = logits.shape
    x, m, s, p, d, ex, q = reference(logits, scale)
    l = (m + torch.log(s))[:, 0]
    W = (p * d).sum(1)
    h = torch.log(s)[:, 0] - W
    pq = (p * q).sum(1)
    tol_l = pq + 4 * EPS * (l.abs() + m[:, 0].abs())
    tol_h = pq + (p * d.abs() * (q + pq[:, None])).sum(1) + (p * ex).sum(1) + 6 * EPS * (torch.log(s)[:, 0].abs() + W.abs())
    within(lse, l, tol_l, "lse")
    within(H, h, tol_h, "entropy")
    if tokens is not None:
        used = (tokens >= 0) & (tokens < V)
        xt = torch.gather(x, 1, torch.where(used, tokens, 0).long())
        want = torch.where(used, xt - l[:, None], 0.0)
        size = torch.where(torch.isfinite(xt), xt.abs(), 0.0)
        within(logp, want, tol_l[:, None] + 4 * EPS * (size + l.abs()[:, None]), "logp")
    if k:
        order = torch.sort(logits.double(), dim=1, descending=True, stable=True).indices[:, :k]
        n = min(k, V)
        assert torch.equal(top[:, :n], order.to(torch.int32))
        xt = torch.gather(x, 1, order)
        size = torch.where(torch.isfinite(xt), xt.abs(), 0.0)
        within(top_logp[:, :n], xt - l[:, None], tol_l[:, None] + 4 * EPS * (size + l.abs()[:, None]), "top_logp")
        assert (top[:, n:] == -1).all() and (top_logp[:, n:] == -math.inf).all()


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("rows,V,T,k", [(1, 1, 1, 1), (3, 2, 4, 5), (2, 7, 0, 0), (5, 63, 5, 3), (4, 64, 1, 64), (3, 65, 100, 65),
                                        (1, 1000, 1024, 128), (9, 4097, 7, 20), (70, 8191, 3, 50), (2, 8193, 4, 1), (300, 513, 2, 10),
                                        (1, 50021, 4, 50), (33, 50021, 10, 128), (1, 131072, 1, 20), (3, 262144, 5, 64),
                                        (20000, 17, 1, 2), (700, 9000, 1, 0), (600, 12289, 4, 33)])
def test_values_and_alternatives(rows, V, T, k, type):
    import paper_1704_07355_amd as Q
    for masked, scale in ((0.0, 1.0), (0.6, 0.75)):
        logits = make(rows, V, type, rows + V, masked)
        logits[:, V // 2] = 1.5  # something is left in every row
        tokens = make_tokens(rows, V, T, V) if T else None
        check(Q.qadc_token_logprobs(logits, tokens, k, scale), logits, tokens, k, scale)


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("V", [100, 5000, 40003])
def test_ties_go_to_the_lowest_token(V, type):
    import paper_1704_07355_amd as Q
    g = gen(V)
    rows = 6
    few = torch.randint(-2, 3, (rows, V), generator=g, device=DEV).to(TYPES[type])
    few[1] = 0.0
    few[2] = torch.where(torch.rand((V,), generator=g, device=DEV) < 0.5, 0.0, -0.0).to(TYPES[type])  # equal zeros
    few[3] = -math.inf
    few[3, V - 3:] = 1.0
    for k in (1, 64, 100):
        check(Q.qadc_token_logprobs(few, None, k), few, None, k, 1.0)


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("order", ["ascending", "descending", "last", "one in a thousand"])
def test_orders_in_which_bounds_come_late(order, type):
    import paper_1704_07355_amd as Q
    for rows, V in ((1, 60000), (400, 30000)):
        x = make(rows, V, type, 3)
        if order != "last" and order != "one in a thousand":
            x = torch.sort(x, dim=1, descending=order == "descending").values
        elif order == "last":
            x[:, V - 200:] += 20.0
        else:
            x[:, ::1000] += 20.0
        check(Q.qadc_token_logprobs(x, None, 100), x, None, 100, 1.0)


@pytest.mark.parametrize("type", list(TYPES))
def test_rows_that_a_mask_leaves_empty_and_rows_that_are_not_finite(type):
    import paper_1704_07355_amd as Q
    for rows, V in ((8, 300), (8, 70000)):
        x = make(rows, V, type, 9)
        tokens = make_tokens(rows, V, 6, 4)
        clean = Q.qadc_token_logprobs(x, tokens, 10)
        x[1] = -math.inf
        x[3, V // 3] = math.nan
        x[4, V // 2] = math.inf
        x[5, 5] = TYPES[type] is torch.float16 and -65504.0 or torch.finfo(TYPES[type]).min  # a mask of the type's lowest value
        x[6] = -math.inf
        x[6, V - 1] = 2.0
        got = Q.qadc_token_logprobs(x, tokens, 10)
        logp, lse, H, top, top_logp = got
        used = (tokens >= 0) & (tokens < V)
        assert lse[1] == -math.inf and H[1] == 0 and (top_logp[1] == -math.inf).all()
        assert (logp[1][used[1]] == -math.inf).all() and (logp[1][~used[1]] == 0).all()
        assert torch.equal(top[1], torch.arange(10, device=DEV, dtype=torch.int32))
        for r, v in ((3, V // 3), (4, V // 2)):
            assert torch.isnan(lse[r]) and torch.isnan(H[r]) and torch.isnan(logp[r][used[r]]).all() and top[r, 0] == v
            assert torch.equal(top[r], torch.sort(x[r].double(), descending=True, stable=True).indices[:10].to(torch.int32))
        assert lse[6] == 2.0 and H[6] == 0.0 and top[6, 0] == V - 1 and top_logp[6, 0] == 0.0
        assert torch.equal(top[6, 1:], torch.arange(9, device=DEV, dtype=torch.int32))
        keep = [0, 2, 7]
        assert all(torch.equal(a[keep], b[keep]) for a, b in zip(got, clean))
        check([t[5:6] for t in got], x[5:6], tokens[5:6], 10, 1.0)
        # the gradient: nothing for the empty row, NaN where the sum is, and finite elsewhere
        dl = torch.ones((rows, 6), device=DEV)
        dx = Q.qadc_token_logprobs_backward(x, tokens, lse, H, dl, torch.ones((rows,), device=DEV))
        assert not dx[1].any() and torch.isnan(dx[[3, 4]]).any(1).all() and torch.isfinite(dx[[0, 2, 5, 6, 7]]).all()


def check_grad(dx, logits, tokens, lse, H, dlogp, dH, scale, type):
    rows, V = logits.shape
    x = logits.double() * scale
    lp = x - lse.double()[:, None]
    p = torch.exp(lp)
    lz = torch.where(p > 0, lp, 0.0)
    used = (tokens >= 0) & (tokens < V) if tokens is not None else None
    own = torch.zeros_like(x)
    total = size = torch.zeros((rows, 1), dtype=torch.float64, device=DEV)
    T = 0
    if tokens is not None:
        T = tokens.shape[1]
        dl = torch.where(used, dlogp, 0.0).double()
        own.scatter_add_(1, torch.where(used, tokens, 0).long(), dl)
        total, size = dl.sum(1, keepdim=True), dl.abs().sum(1, keepdim=True)
    g = torch.zeros((rows, 1), dtype=torch.float64, device=DEV) if dH is None else dH.double()[:, None]
    h = torch.zeros_like(g) if dH is None else H.double()[:, None]
    inner = total + g * (lz + h)
    want = scale * (own - p * inner)
    q = 6 * EPS * (torch.where(p > 0, x, 0.0).abs() + lse.double().abs()[:, None]) + 8 * EPS
    tol = p * (q * inner.abs() + (T + 4) * EPS * size + 4 * EPS * g.abs() * (lz.abs() + h.abs() + lse.double().abs()[:, None]))
    tol = scale * (tol + (T + 4) * EPS * torch.where(own != 0, size, 0.0)) + 4 * EPS * want.abs()
    within(dx, want, tol * (1 + UNIT[type]) + UNIT[type] * want.abs() + LEAST[type] + 2.0 ** -126, "dlogits")


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("rows,V,T", [(1, 1, 1), (3, 2, 5), (5, 63, 4), (2, 300, 0), (3, 1000, 1024), (9, 4097, 7), (40, 8191, 1),
                                      (1, 131072, 4), (2, 262144, 30), (9000, 17, 1), (300, 9001, 1), (1030, 2048, 2)])
def test_gradient(rows, V, T, type):
    import paper_1704_07355_amd as Q
    g = gen(rows * V)
    logits = make(rows, V, type, V, 0.2)
    logits[:, V // 2] = 1.0
    tokens = make_tokens(rows, V, T, 2) if T else None
    dl = torch.randn((rows, T), generator=g, device=DEV) if T else None
    for dH, scale in ((None, 1.0), (torch.randn((rows,), generator=g, device=DEV), 1.5)):
        _, lse, H, _, _ = Q.qadc_token_logprobs(logits, tokens, 0, scale)
        dx = Q.qadc_token_logprobs_backward(logits, tokens, lse, H, dl, dH, scale)
        check_grad(dx, logits, tokens, lse, H, dl, dH, scale, type)


def test_gradient_by_differences():
    """Central differences with h = 2^-6 along the gradient: off by h^2 / 6 times the third derivative and by the rounding of the
    sum of some log probabilities, 2^-21 each, over h."""
    import paper_1704_07355_amd as Q
    rows, V, T, scale = 5, 700, 6, 1.25
    g = gen(1)
    x = make(rows, V, "f32", 11)
    tokens = make_tokens(rows, V, T, 5)
    dl, dH = torch.randn((rows, T), generator=g, device=DEV), torch.randn((rows,), generator=g, device=DEV)

    def loss(x):
        logp, _, H, _, _ = Q.qadc_token_logprobs(x, tokens, 0, scale)
        return ((logp.double() * dl.double()).sum() + (H.double() * dH.double()).sum()).item()

    _, lse, H, _, _ = Q.qadc_token_logprobs(x, tokens, 0, scale)
    dx = Q.qadc_token_logprobs_backward(x, tokens, lse, H, dl, dH, scale)
    e = dx / dx.abs().max()
    h = 2.0 ** -6
    got, want = (dx.double() * e.double()).sum().item(), (loss(x + h * e) - loss(x - h * e)) / (2 * h)
    weight = (dl.abs().sum() + dH.abs().sum()).item()
    assert abs(got - want) <= 4 * h * h * weight + 2.0 ** -21 * 16 * weight / h, (got, want)


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("rows,V,ld,shift", [(1, 333, 333, 1), (5, 1000, 1001, 3), (7, 20001, 20010, 5), (200, 129, 160, 1)])
def test_rows_apart_unaligned_and_in_place(rows, V, ld, shift, type):
    import paper_1704_07355_amd as Q
    x = make(rows, V, type, 2, 0.1)
    x[:, 0] = 0.0
    tokens = make_tokens(rows, V, 8, 3)
    far = apart(x, ld, shift)
    a, b = Q.qadc_token_logprobs(x, tokens, 40), Q.qadc_token_logprobs(far, tokens, 40)
    assert torch.equal(a[3], b[3])
    check(b, x, tokens, 40, 1.0)
    dl, dH = torch.randn((rows, 8), generator=gen(4), device=DEV), torch.ones((rows,), device=DEV)
    want = Q.qadc_token_logprobs_backward(x, tokens, a[1], a[2], dl, dH)
    check_grad(want, x, tokens, a[1], a[2], dl, dH, 1.0, type)
    out = apart(torch.zeros_like(x), ld + 1, shift + 1)
    assert torch.equal(Q.qadc_token_logprobs_backward(far, tokens, a[1], a[2], dl, dH, out=out), want)
    between = torch.as_strided(out, (rows, ld + 1), (ld + 1, 1))[:-1, V:]
    assert torch.isnan(between).all()
    assert torch.equal(Q.qadc_token_logprobs_backward(far, tokens, a[1], a[2], dl, dH, out=far), want)
    assert torch.isnan(torch.as_strided(far, (rows, ld), (ld, 1))[:-1, V:]).all()


def test_one_workspace_for_many_calls_streams_and_equal_bits():
    import paper_1704_07355_amd as Q
    for rows, V, k in ((1, 131072, 20), (3, 40000, 64), (500, 20000, 8)):
        ws = Q.qadc_workspace_init(torch.empty((max(256, Q.qadc_token_logprobs_workspace_bytes(rows, V, k)),), dtype=torch.uint8,
                                               device=DEV))
        x = [make(rows, V, "bf16", s) for s in (1, 2)]
        want = [Q.qadc_token_logprobs(v, None, k) for v in x]
        for _ in range(5):
            for v, w in zip(x, want):
                got = Q.qadc_token_logprobs(v, None, k, workspace=ws)
                assert all(torch.equal(a, b) for a, b in zip(got, w))
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            got = Q.qadc_token_logprobs(x[0], None, k, workspace=ws)
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want[0]))


def test_a_captured_graph_replays():
    import paper_1704_07355_amd as Q
    rows, V, k = 2, 60000, 30
    ws = Q.qadc_workspace_init(torch.empty((max(256, Q.qadc_token_logprobs_workspace_bytes(rows, V, k)),), dtype=torch.uint8,
                                           device=DEV))
    x = make(rows, V, "f16", 1)
    tokens = make_tokens(rows, V, 4, 1)
    Q.qadc_token_logprobs(x, tokens, k, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = Q.qadc_token_logprobs(x, tokens, k, workspace=ws)
    for seed in (3, 4, 5):
        x.copy_(make(rows, V, "f16", seed))
        graph.replay()
        torch.cuda.synchronize()
        check(got, x, tokens, k, 1.0)
        want = Q.qadc_token_logprobs(x, tokens, k)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_offsets_beyond_32_bits():
    import paper_1704_07355_amd as Q
    x = make(3, 5000, "bf16", 6)
    tokens = make_tokens(3, 5000, 4, 6)
    ld = 1_500_000_000
    far = torch.as_strided(torch.empty((2 * ld + 5000,), dtype=torch.bfloat16, device=DEV), (3, 5000), (ld, 1))
    far.copy_(x)
    want, got = Q.qadc_token_logprobs(x, tokens, 9), Q.qadc_token_logprobs(far, tokens, 9)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    dl = torch.ones((3, 4), device=DEV)
    want = Q.qadc_token_logprobs_backward(x, tokens, got[1], got[2], dl)
    Q.qadc_token_logprobs_backward(far, tokens, got[1], got[2], dl, out=far)
    assert torch.equal(far, want)


def test_no_rows_and_refusals_of_the_binding():
    import paper_1704_07355_amd as Q
    x = make(4, 100, "f16", 1)
    tokens = make_tokens(4, 100, 5, 1)
    got = Q.qadc_token_logprobs(x[:0], tokens[:0], 3)
    assert [tuple(t.shape) for t in got] == [(0, 5), (0,), (0,), (0, 3), (0, 3)]
    logp, lse, H, _, _ = Q.qadc_token_logprobs(x, tokens)
    assert Q.qadc_token_logprobs_backward(x[:0], tokens[:0], lse[:0], H[:0], logp[:0]).shape == (0, 100)
    for bad in (lambda: Q.qadc_token_logprobs(x.double()), lambda: Q.qadc_token_logprobs(x.t()), lambda: Q.qadc_token_logprobs(x, tokens[:3]),
                lambda: Q.qadc_token_logprobs(x, tokens.long()), lambda: Q.qadc_token_logprobs(x.cpu(), tokens),
                lambda: Q.qadc_token_logprobs_backward(x, tokens, lse[:3], H, logp),
                lambda: Q.qadc_token_logprobs_backward(x, tokens, lse, None, logp, lse),
                lambda: Q.qadc_token_logprobs_backward(x, tokens, lse, H, logp[:, :4].contiguous()),
                lambda: Q.qadc_token_logprobs_backward(x, tokens, lse, H, logp, out=torch.empty((4, 100), device=DEV))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: Q.qadc_token_logprobs(x, tokens, 129), lambda: Q.qadc_token_logprobs(x, tokens, 1, 0.0),
                lambda: Q.qadc_token_logprobs(x, tokens, 1, float("inf"))):
        with pytest.raises(Q.QadcError):
            bad()


@pytest.mark.parametrize("k", [0, 20])
@pytest.mark.parametrize("rows,V", [(400, 131072), (410, 60000), (1000, 20000), (5, 400000)])
def test_a_workspace_for_a_batch_serves_its_smaller_batches(rows, V, k):
    import paper_1704_07355_amd as Q
    ws = torch.empty((Q.qadc_token_logprobs_workspace_bytes(rows, V, k),), dtype=torch.uint8, device=DEV)
    x = make(rows, V, "bf16", 31)
    for n in (rows, 399, 130, 3, 1):
        if n > rows:
            continue
        got, want = Q.qadc_token_logprobs(x[:n], None, k, workspace=ws), Q.qadc_token_logprobs(x[:n], None, k)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), n


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("rows,V", [(3, 900), (2, 131072), (420, 700)])
@pytest.mark.parametrize("offset,scale", [(1000.0, 1.0), (-3000.0, 0.75), (100.0, 1e3)])
def test_log_probabilities_do_not_take_on_the_offset(offset, scale, rows, V, type):
    """x - lse is scale (logit - m) - log s: the difference of two logits, a product and a difference, however large both are."""
    import paper_1704_07355_amd as Q
    logits = (make(rows, V, "f32", 21) + offset).to(TYPES[type])
    tokens = make_tokens(rows, V, 5, 22)
    tokens[:, 4] = logits.argmax(1).to(torch.int32)
    logp, _, _, top, top_logp = Q.qadc_token_logprobs(logits, tokens, 6, scale)
    x = logits.double() * scale
    m = x.max(1, keepdim=True).values
    d = x - m
    s = torch.exp(d).sum(1, keepdim=True)
    p = torch.exp(d) / s
    off = 6 * EPS * d.abs() + (V / 256 + 44) * EPS           # of an exponential and of the sum up to it, relative
    tol_s = (p * off).sum(1, keepdim=True) + 4 * EPS * torch.log(s)
    used = (tokens >= 0) & (tokens < V)
    at = torch.where(used, tokens, 0).long()
    dt = torch.gather(d, 1, at)
    within(logp, torch.where(used, dt - torch.log(s), 0.0), tol_s + 4 * EPS * dt.abs(), "logp")
    order = torch.sort(logits.double(), dim=1, descending=True, stable=True).indices[:, :6]
    dt = torch.gather(d, 1, order)
    assert torch.equal(top, order.to(torch.int32))
    within(top_logp, dt - torch.log(s), tol_s + 4 * EPS * dt.abs(), "top_logp")


@pytest.mark.parametrize("V", [300, 70000])
def test_log_probabilities_where_the_scaled_logit_passes_a_float(V):
    """A finite row whose scale * logit is no float32: the likeliest token has all, lse is NaN (not the -inf of an empty row),
    and so is the gradient that would need it."""
    import paper_1704_07355_amd as Q
    for sign in (1.0, -1.0):
        logits = -sign * torch.rand((4, V), generator=gen(V), device=DEV) + (0.0 if sign > 0 else -1000.0)
        logits[:, 7] = 500.0 if sign > 0 else -500.0
        logits[3] = -math.inf
        tokens = torch.tensor([[7, 8]], device=DEV, dtype=torch.int32).expand(4, 2).contiguous()
        logp, lse, H, top, top_logp = Q.qadc_token_logprobs(logits, tokens, 2, 1e38)
        assert (logp[:3, 0] == 0).all() and (logp[:3, 1] == -math.inf).all() and not H.any()
        assert (top[:3, 0] == 7).all() and (top_logp[:3, 0] == 0).all() and (top_logp[:3, 1] == -math.inf).all()
        assert torch.isnan(lse[:3]).all() and lse[3] == -math.inf and (logp[3] == -math.inf).all()
        dx = Q.qadc_token_logprobs_backward(logits, tokens, lse, H, torch.ones((4, 2), device=DEV), None, 1e38)
        assert torch.isnan(dx[:3]).all() and not dx[3].any()
        logp, lse, H, _, _ = Q.qadc_token_logprobs(logits, tokens, 0, 1e3)
        assert (logp[:3, 0] == 0).all() and torch.isfinite(lse[:3]).all() and torch.isfinite(logp[:3]).all()


def usable_rows(rows, V, type, which, lowest):
    """Logits of which a grammar leaves few, or many of one value: (logits, the place of what is left)."""
    x = make(rows, V, type, 51)
    t = torch.arange(V, device=DEV)
    left = {"five": (t % (V // 5)) == 17, "range of 200": (t >= V // 3) & (t < V // 3 + 200),
            "range of 2000": (t >= V // 2 + 1) & (t < V // 2 + 2001), "first token": t == 0, "last token": t == V - 1,
            # of every workgroup's worth of logits the same few threads': more of them than a list holds
            "a few threads'": (t // 8) % 256 < 20}[which]
    return torch.where(left, x, torch.finfo(TYPES[type]).min if lowest else -math.inf).to(TYPES[type])


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("lowest", [False, True])
@pytest.mark.parametrize("which", ["five", "range of 200", "range of 2000", "first token", "last token", "a few threads'"])
@pytest.mark.parametrize("rows,V", [(1, 131072), (2, 60000), (401, 60000), (3, 500)])
def test_alternatives_of_masked_rows(rows, V, which, lowest, type):
    import paper_1704_07355_amd as Q
    if V < 10000 and which.startswith("range of 2000"):
        V = 5000
    x = usable_rows(rows, V, type, which, lowest)
    for k in (50, 128):
        check(Q.qadc_token_logprobs(x, None, k), x, None, k, 1.0)


@pytest.mark.parametrize("type", list(TYPES))
def test_alternatives_of_rows_cut_off_below_and_above(type):
    """Many logits of one value where the k-th lies: the first of them in the row are taken, wherever they begin."""
    import paper_1704_07355_amd as Q
    for rows, V in ((1, 131072), (401, 60000)):
        x = make(rows, V, type, 52)
        above = torch.clamp(x, max=2.0)
        below = torch.where(torch.arange(V, device=DEV) < V // 2, x - 100.0, 3.0).to(TYPES[type])
        below[:, V // 2 + 100::V // 64] = 4.0
        odd = below.clone()
        odd[:, 3] = math.nan
        for k in (20, 128):
            for y in (above, below):
                check(Q.qadc_token_logprobs(y, None, k), y, None, k, 1.0)
            top = Q.qadc_token_logprobs(odd, None, k)[3]
            want = torch.sort(odd.double(), dim=1, descending=True, stable=True).indices[:, :k]
            assert torch.equal(top, want.to(torch.int32))
