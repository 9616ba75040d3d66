"""Neighbours' tokens mixed into log probabilities, against the formula in 64 bits.

Tolerances, with e = 2^-24: an exponent v = -beta step (d - min d) is off by at most 4 e |v|, a sum of R exponentials by (R + 8) e
relative and its logarithm by that; log P by twice that and its own rounding, the mixture by the larger of its two terms' errors.
"""

import math

import pytest

import torch

from lm_common import DEV, EPS, gen, within

pytestmark = pytest.mark.gpu


def make(rows, R, T, n, kind, seed, vocabulary=50):
    g = gen(seed)
    values = torch.randint(0, vocabulary, (n,), generator=g, device=DEV, dtype=torch.int32)
    ids = torch.randint(0, n, (rows, R), generator=g, device=DEV, dtype=torch.int32)
    if R > 4:
        ids[::3, R // 2:] = -1
    if kind == "u8":
        dist = torch.randint(0, 256, (rows, R), generator=g, device=DEV, dtype=torch.uint8)
        step = 0.5 + torch.rand((rows,), generator=g, device=DEV)
    else:
        dist, step = 100.0 + 100.0 * torch.rand((rows, R), generator=g, device=DEV), None
    tokens = torch.randint(-1, vocabulary + 5, (rows, T), generator=g, device=DEV, dtype=torch.int32)
    lm = -10.0 * torch.rand((rows, T), generator=g, device=DEV)
    return ids, dist, values, tokens, lm, step


def check(got, ids, dist, values, tokens, lm, lam, beta, step):
    mix, knn = got
    rows, R = ids.shape
    n = values.numel()
    id64 = ids.long() & 0xFFFFFFFF
    used = (id64 < n) & torch.isfinite(dist.float())
    value = torch.where(used, values[torch.where(used, id64, 0)].long(), -5)
    d = dist.double() * (1.0 if step is None else step.double()[:, None])
    v = torch.where(used, -beta * d, -math.inf)
    top = v.max(1, keepdim=True).values
    any_ = torch.isfinite(top)
    v = torch.where(used, v - torch.where(any_, top, 0.0), -math.inf)
    log_z = torch.logsumexp(v, 1, keepdim=True)
    votes = value[:, None, :] == tokens[:, :, None]
    log_p = torch.logsumexp(torch.where(votes, v[:, None, :], -math.inf), 2) - torch.where(any_, log_z, 0.0)
    log_p = torch.where(any_, log_p, -math.inf)
    a = lm.double() + (math.log1p(-lam) if lam < 1 else -math.inf)
    b = log_p + (math.log(lam) if lam > 0 else -math.inf)
    want = torch.where(any_, torch.logaddexp(a, b), lm.double())
    off = tokens < 0
    size = torch.where(used, v.abs(), 0.0).max(1, keepdim=True).values
    tol_p = (2 * R + 32) * EPS + 8 * EPS * size + 4 * EPS * torch.where(torch.isfinite(log_p), log_p, 0.0).abs()
    within(knn, torch.where(off, 0.0, log_p), tol_p, "knn")
    within(mix, torch.where(off, 0.0, want), tol_p + 8 * EPS * (1 + torch.where(torch.isfinite(want), want, 0.0).abs() + lm.double().abs()), "mix")


@pytest.mark.parametrize("kind", ["u8", "f32"])
@pytest.mark.parametrize("rows,R,T,n", [(1, 1, 1, 1), (1, 100, 120, 5000), (3, 7, 5, 10), (5, 64, 64, 100), (2, 65, 300, 1000), (40, 256, 3, 999),
                                        (7, 1000, 1, 5000), (9, 1024, 130, 20), (3000, 33, 2, 100), (2, 1023, 1100, 100000), (4, 16, 0, 10)])
def test_mixture(rows, R, T, n, kind):
    import paper_1704_07355_amd as Q
    ids, dist, values, tokens, lm, step = make(rows, R, T, n, kind, rows + R)
    for lam, beta in ((0.25, 0.05), (0.0, 0.1), (1.0, 0.01), (0.5, 0.0)):
        check(Q.qadc_neighbour_mix(ids, dist, values, tokens, lm, lam, beta, step), ids, dist, values, tokens, lm, lam, beta, step)


@pytest.mark.parametrize("R", [5, 64, 300, 1024])
def test_rows_without_neighbours_and_neighbours_left_out(R):
    import paper_1704_07355_amd as Q
    ids, dist, values, tokens, lm, _ = make(6, R, 20, 50, "f32", R)
    ids[0] = -1                      # none
    ids[1] = 50                      # all beyond the stored states
    dist[2] = math.inf               # no finite distance
    dist[3, 0], dist[3, 1] = math.nan, -math.inf
    ids[4, 1:] = -1                  # one neighbour
    ids[5] = 3                       # one stored state many times
    lm[5, 3] = -math.inf             # a masked token
    got = Q.qadc_neighbour_mix(ids, dist, values, tokens, lm, 0.3, 0.1)
    check(got, ids, dist, values, tokens, lm, 0.3, 0.1, None)
    live = tokens[:3] >= 0
    assert torch.equal(got[0][:3][live], lm[:3][live]) and (got[1][:3][live] == -math.inf).all()
    # no stored state at all
    mix, knn = Q.qadc_neighbour_mix(ids, dist, values[:0], tokens, lm, 0.3, 0.1)
    live = tokens >= 0
    assert torch.equal(mix[live], lm[live]) and (knn[live] == -math.inf).all() and not mix[~live].any()


def test_weights_below_the_smallest_float():
    """Votes e^-200 and e^-1000 behind the nearest, and a model's log probability of -500: all still there."""
    import paper_1704_07355_amd as Q
    ids = torch.arange(4, device=DEV, dtype=torch.int32)[None, :].contiguous()
    dist = torch.tensor([[0.0, 200.0, 1000.0, 1000.0]], device=DEV)
    values = torch.tensor([1, 2, 3, 3], device=DEV, dtype=torch.int32)
    tokens = torch.tensor([[1, 2, 3, 4]], device=DEV, dtype=torch.int32)
    lm = torch.tensor([[-500.0, -500.0, -500.0, -500.0]], device=DEV)
    got = Q.qadc_neighbour_mix(ids, dist, values, tokens, lm, 0.5, 1.0)
    check(got, ids, dist, values, tokens, lm, 0.5, 1.0, None)
    assert torch.isfinite(got[1][0, :3]).all() and got[1][0, 3] == -math.inf


def test_distances_further_apart_than_a_float_reaches():
    """With beta 0 all neighbours weigh the same, also where the difference of two distances overflows."""
    import paper_1704_07355_amd as Q
    ids = torch.arange(4, device=DEV, dtype=torch.int32)[None, :].contiguous()
    dist = torch.tensor([[-3e38, 3e38, 0.0, 1.0]], device=DEV)
    values = torch.tensor([1, 2, 2, 2], device=DEV, dtype=torch.int32)
    tokens = torch.tensor([[1, 2, 3]], device=DEV, dtype=torch.int32)
    lm = torch.tensor([[-1.0, -2.0, -3.0]], device=DEV)
    check(Q.qadc_neighbour_mix(ids, dist, values, tokens, lm, 0.5, 0.0), ids, dist, values, tokens, lm, 0.5, 0.0, None)


def test_results_of_a_search_streams_and_equal_bits():
    import paper_1704_07355_amd as Q
    ids, dist, values, tokens, lm, step = make(50, 100, 30, 1000, "u8", 7)
    want = Q.qadc_neighbour_mix(ids, dist, values, tokens, lm, 0.2, 0.02, step)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = Q.qadc_neighbour_mix(ids.view(torch.uint32), dist, values, tokens, lm, 0.2, 0.02, step)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # on their own: a row's result does not depend on the rows beside it
    one = Q.qadc_neighbour_mix(ids[7:8], dist[7:8], values, tokens[7:8], lm[7:8], 0.2, 0.02, step[7:8])
    assert all(torch.equal(a[0], b[7]) for a, b in zip(one, want))


def test_refusals_of_the_binding():
    import paper_1704_07355_amd as Q
    ids, dist, values, tokens, lm, step = make(5, 20, 4, 100, "u8", 1)
    f = lambda **k: Q.qadc_neighbour_mix(**{**dict(ids=ids, dist=dist, values=values, tokens=tokens, lm_logp=lm, lam=0.5, beta=1.0, step=step), **k})
    f()
    for bad in (dict(ids=ids.long()), dict(dist=dist[:, :19]), dict(dist=dist.int()), dict(values=values.long()), dict(tokens=tokens[:4]),
                dict(lm_logp=lm[:, :3]), dict(step=step[:4]), dict(lm_logp=lm.half()), dict(ids=ids.cpu())):
        with pytest.raises(ValueError):
            f(**bad)
    for bad in (dict(lam=-0.1), dict(lam=1.5), dict(lam=float("nan")), dict(beta=-1.0), dict(beta=float("inf"))):
        with pytest.raises(Q.QadcError):
            f(**bad)
    wide = torch.zeros((1, 1025), dtype=torch.int32, device=DEV)
    with pytest.raises(Q.QadcError):
        Q.qadc_neighbour_mix(wide, wide.float(), values, tokens[:1], lm[:1], 0.5, 1.0)


def test_weights_whose_product_passes_a_float():
    """beta and step are finite, their product is not: the nearest still have their votes, and a difference that the product brings
    back to order one still counts.  The same for a difference that passes a float where beta brings it back."""
    import paper_1704_07355_amd as Q
    ids = torch.arange(4, device=DEV, dtype=torch.int32)[None, :].expand(3, 4).contiguous()
    values = torch.tensor([1, 2, 1, 3], device=DEV, dtype=torch.int32)
    tokens = torch.tensor([[1, 2, 3, 4, -1]], device=DEV, dtype=torch.int32).expand(3, 5).contiguous()
    lm = -torch.arange(1.0, 16.0, device=DEV).reshape(3, 5)
    step = torch.tensor([2.0 ** 100, 2.0 ** 90, 1.0], device=DEV)
    near = torch.full((3, 4), 7, device=DEV, dtype=torch.uint8)
    check(Q.qadc_neighbour_mix(ids, near, values, tokens, lm, 0.5, 2.0 ** 60, step), ids, near, values, tokens, lm, 0.5, 2.0 ** 60, step)
    near[:, 3] = 9  # e^(-2^161): no vote is left
    knn = Q.qadc_neighbour_mix(ids, near, values, tokens, lm, 0.5, 2.0 ** 60, step)[1]
    want = torch.tensor([2 / 3, 1 / 3], device=DEV, dtype=torch.float64).log().expand(2, 2)
    within(knn[:2, :2], want, 64 * EPS)
    assert (knn[:2, 2:4] == -math.inf).all() and not knn[:, 4].any()
    tiny = torch.tensor([[0.0, 1.0, 2.0, 0.5]]) * 2.0 ** -140
    tiny = torch.cat((tiny, tiny * 2.0 ** 5, tiny), 0).to(DEV)
    step = torch.tensor([2.0 ** 80, 2.0 ** 75, 2.0 ** 80], device=DEV)
    check(Q.qadc_neighbour_mix(ids, tiny, values, tokens, lm, 0.5, 2.0 ** 60, step), ids, tiny, values, tokens, lm, 0.5, 2.0 ** 60, step)
    far = torch.tensor([[-3e38, 3e38, 0.0, 1e38]], device=DEV).expand(3, 4).contiguous()
    check(Q.qadc_neighbour_mix(ids, far, values, tokens, lm, 0.5, 2.0 ** -126, None), ids, far, values, tokens, lm, 0.5, 2.0 ** -126, None)


@pytest.mark.parametrize("rows,R,T", [(2047, 100, 20), (2047, 256, 64), (3000, 300, 20), (3000, 100, 65), (2500, 1024, 3)])
def test_rows_alone_give_the_bits_they_give_among_others(rows, R, T):
    import paper_1704_07355_amd as Q
    for kind in ("u8", "f32"):
        ids, dist, values, tokens, lm, step = make(rows, R, T, 5000, kind, 8)
        want = Q.qadc_neighbour_mix(ids, dist, values, tokens, lm, 0.2, 0.02, step)
        for r in (0, 1, rows - 1):
            one = slice(r, r + 1)
            got = Q.qadc_neighbour_mix(ids[one], dist[one], values, tokens[one], lm[one], 0.2, 0.02, None if step is None else step[one])
            assert all(torch.equal(p[0], q[r]) for p, q in zip(got, want))
