"""Distillation from a teacher's stored tokens against its definition in 64 bits.

Tolerances, from the arithmetic (u: half a unit in the last place of the output's type, e = 2^-24): a sum of V exponentials has
chains of at most V/400 + 33 additions; each exponential 2^t is off by 2 |t| e and 3 e, and over a row sum 2^t |t| / sum 2^t is at
most log2 V + 2.  So sums, and with them lse, are off by E = (V/400 + 36 + 2 (log2 V + 2)) e relative; log Q, from the quotient of two of
them, by 2 E.  A probability from a given lse is off by (3 |log q| + 8) e: the argument's sum, the difference to log Q and its
product with log2(e) are rounded, each off by at most |log q| e.
"""

import math

import pytest

import torch

from lm_common import DEV, EPS, LEAST, TYPES, UNIT, apart, gen, within

pytestmark = pytest.mark.gpu


def _error(V):
    return (V / 400 + 36 + 2 * (math.log2(V) + 2)) * EPS


def _inputs(rows, V, k, type, seed, noise=0.7, scale=1.0):
    g = gen(seed)
    x = (2.5 * torch.randn((rows, V), generator=g, device=DEV)).to(TYPES[type])
    t = scale * x.float() + noise * torch.randn((rows, V), generator=g, device=DEV)
    n = min(k, V)
    lp, at = torch.topk(torch.log_softmax(t, 1), n, dim=1)
    idx = torch.full((rows, k), -1, dtype=torch.int32, device=DEV)
    logp = torch.full((rows, k), -math.inf, device=DEV)
    idx[:, :n], logp[:, :n] = at.to(torch.int32), lp
    if k > 3:  # unused slots anywhere: what their log probabilities are is not looked at
        idx[::3, 1], logp[::3, 1] = -1, math.nan
        idx[1::3, 2], logp[1::3, 2] = V, 5.0
    w = torch.rand((rows,), generator=g, device=DEV) - 0.3
    w[rows // 2] = 0.0 if rows > 1 else 0.5
    return x, idx, logp, w


def _reference(x, idx, logp, scale, tail):
    """loss, lse, log Q, and what the gradient needs, all in 64 bits."""
    V = x.shape[1]
    x = x.double() * torch.tensor(scale, dtype=torch.float32).item()
    lse = torch.logsumexp(x, 1)
    used = (idx >= 0) & (idx < V)
    at = torch.where(used, idx, V).long()
    p = torch.where(used, torch.exp(logp.double()), 0.0)
    P = p.sum(1)
    rest = (1 - P).clamp(min=0.0) if tail else torch.zeros_like(P)
    log_p = logp.double().masked_fill(~used, 0.0)
    if not tail:
        log_p = torch.where(P > 0, log_p.t() - torch.log(P), 0.0).t()
        p = torch.where(P > 0, p.t() / P, 0.0).t()
    wide = torch.cat((x, torch.full_like(x[:, :1], -math.inf)), 1)
    xt = torch.gather(wide, 1, at)
    inside = torch.zeros_like(wide, dtype=torch.bool).scatter_(1, at, True)
    log_tail = torch.logsumexp(wide.masked_fill(inside, -math.inf), 1) - lse
    log_tail = torch.where(lse == -math.inf, -math.inf, log_tail)
    rest = torch.where(log_tail == -math.inf, 0.0, rest)
    log_q = torch.where((lse == -math.inf)[:, None], -math.inf, xt - lse[:, None])
    loss = torch.where(p > 0, p * (log_p - log_q), 0.0).sum(1) + torch.where(rest > 0, rest * (torch.log(rest) - log_tail), 0.0)
    T = P + rest if tail else (P > 0).double()
    want = torch.zeros_like(wide).scatter_add_(1, at, p)[:, :V]
    return dict(x=x, loss=loss, lse=lse, log_tail=log_tail, P=P, rest=rest, T=T, p=want, inside=inside[:, :V])


def _gradient(ref, lse, log_tail, w, scale):
    """The gradient of given statistics, with the size of its terms."""
    lp = torch.where((lse == -math.inf)[:, None], -math.inf, ref["x"] - lse[:, None])
    q = torch.exp(lp)
    ratio = torch.where(ref["rest"] > 0, ref["rest"] * torch.exp(-log_tail), 0.0)[:, None]
    share = torch.where(ref["inside"], ref["T"][:, None].expand(q.shape), ref["T"][:, None] - ratio)
    dead = (lse == -math.inf) | (w == 0)
    f = (w.double() * scale)[:, None]
    want = torch.where(dead[:, None], 0.0, f * (share * q - ref["p"]))
    return want, lp, q, share, ratio, f.abs()


def _check_gradient(got, ref, lse, log_tail, w, scale, type, E=0.0):
    want, lp, q, share, ratio, f = _gradient(ref, lse, log_tail, w, scale)
    near = (3 * lp.abs().clamp(max=200.0) + 8) * EPS + E
    inner = f * (share.abs() * q * near + torch.where(ref["inside"], 0.0, ratio * q * 2 * E) + 6 * EPS * ref["p"])
    within(got, want, UNIT[type] * want.abs() + LEAST[type] + 2.0 ** -126 + inner * (1 + UNIT[type]), "gradient")


def _check(x, idx, logp, w, scale, tail):
    import paper_1704_07355_amd as Q
    type = [k for k, t in TYPES.items() if t == x.dtype][0]
    ref, E = _reference(x, idx, logp, scale, tail), _error(x.shape[1])
    loss, lse, log_tail = Q.qadc_distill(x, idx, logp, scale, tail)
    tol = 2 * E * (ref["P"] + ref["rest"] + 1) + EPS * (ref["loss"].abs() + ref["rest"] * ref["log_tail"].nan_to_num(neginf=0.0).abs())
    within(loss, ref["loss"], tol, "loss")
    within(lse, ref["lse"], E + 2 * EPS * ref["lse"].abs(), "lse")
    within(log_tail, ref["log_tail"], 2 * E + EPS * ref["log_tail"].abs(), "log Q")
    grad = Q.qadc_distill_backward(x, idx, logp, lse, log_tail, w, scale, tail)
    _check_gradient(grad, ref, lse.double(), log_tail.double(), w, scale, type)
    step_loss, step = Q.qadc_distill_step(x, idx, logp, w, scale, tail)
    within(step_loss, ref["loss"], tol, "loss of the step")
    # (few rows take both calls in turn: lse there is a float32)
    _check_gradient(step, ref, ref["lse"], ref["log_tail"], w, scale, type,
                    2 * E + EPS * ref["lse"].nan_to_num(neginf=0.0).abs().max().item())
    return loss, lse, log_tail, grad, step


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("rows,V,k", [(1, 1, 1), (2, 2, 1), (3, 7, 9), (5, 100, 0), (4, 1000, 128), (2, 8192, 20), (3, 8193, 64), (7, 20011, 5),
                                      (1, 131072, 20), (2, 140001, 100), (130, 1000, 33), (131, 8190, 128), (129, 16500, 3), (140, 33000, 64),
                                      (128, 65536, 64), (130, 65537, 20), (450, 3001, 17), (401, 12000, 1), (128, 131065, 10), (3, 40961, 64), (50, 50021, 20),
                                      (12, 90003, 128)])
def test_loss_and_gradients(rows, V, k, type):
    for tail in (True, False):
        scale = 1.0 if V % 2 else 0.6
        _check(*_inputs(rows, V, k, type, rows + V, scale=scale), scale, tail)


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("rows,V,ld,shift", [(5, 1000, 1003, 1), (3, 9001, 9004, 3), (2, 7, 9, 5), (140, 4000, 4005, 7), (135, 70000, 70001, 1), (6, 41003, 41004, 3)])
def test_rows_apart_and_unaligned(rows, V, ld, shift, type):
    import paper_1704_07355_amd as Q
    x, idx, logp, w = _inputs(rows, V, 20, type, ld)
    wide = apart(x, ld, shift)
    loss, lse, log_tail, grad, step = _check(wide, idx, logp, w, 1.0, True)
    for ld2, shift2 in ((ld + 2, shift + 1), (ld + 8, 0)):
        room = apart(x, ld2, shift2)
        Q.qadc_distill_backward(wide, idx, logp, lse, log_tail, w, out=room)
        assert torch.equal(room, grad)
        assert torch.isnan(torch.as_strided(room, (rows - 1, 2), (ld2, 1), room.storage_offset() + V).float()).all()
        Q.qadc_distill_step(wide, idx, logp, w, out=room)
        assert torch.equal(room, step)
        assert torch.isnan(torch.as_strided(room, (rows - 1, 2), (ld2, 1), room.storage_offset() + V).float()).all()
    for call, want in ((lambda t: Q.qadc_distill_backward(t, idx, logp, lse, log_tail, w, out=t), grad),
                       (lambda t: Q.qadc_distill_step(t, idx, logp, w, out=t)[1], step)):
        assert torch.equal(call(apart(x, ld, shift)), want)  # in place


@pytest.mark.parametrize("rows", [5, 200])
def test_rows_with_little_in_them(rows):
    """Rows of a padded batch, masked students, teachers that store everything or nothing, and a token stored twice."""
    import paper_1704_07355_amd as Q
    V, k = 500, 12
    x, idx, logp, w = _inputs(rows, V, k, "f32", 3)
    x[1:3] = -math.inf                      # nothing left
    x[2, 40] = 1.0                          # one token left, which is not stored
    idx[2, 0], logp[2] = 41, -math.inf
    x[3, :] = -math.inf                     # stored tokens left and, where its unused slot points, token 0
    x[3, idx[3].clamp(min=0, max=V - 1).long()] = torch.arange(k, device=DEV).float()
    idx[4], logp[4] = -1, math.nan          # an empty teacher
    idx[0, 5], idx[0, 6] = idx[0, 4], idx[0, 4]  # a token stored three times
    w[:5] = torch.tensor([0.5, 0.7, -0.4, 0.3, 0.9], device=DEV)
    for tail in (True, False):
        loss, lse, log_tail, grad, step = _check(x, idx, logp, w, 1.0, tail)
        assert lse[1] == log_tail[1] == -math.inf and loss[1] == math.inf and (grad[1] == 0).all() and (step[1] == 0).all()
        assert torch.isfinite(log_tail[3]) and torch.isfinite(loss[3]) and torch.isfinite(grad[3]).all()
        assert loss[4] == 0 if not tail else abs(loss[4].item()) < 1e-6
    # only stored tokens left: the tail's term is left out
    only = torch.full_like(x, -math.inf)
    only[:, 40:40 + k] = torch.randn((rows, k), generator=gen(6), device=DEV)
    at = torch.arange(40, 40 + k, device=DEV, dtype=torch.int32).expand(rows, k).contiguous()
    p = torch.log_softmax(torch.randn((rows, k), generator=gen(7), device=DEV), 1) - 0.1
    for tail in (True, False):
        loss, _, log_tail, _, _ = _check(only, at, p, w, 1.0, tail)
        assert (log_tail == -math.inf).all() and torch.isfinite(loss).all()
    # a stored token that the student's mask excludes
    x, idx, logp, w = _inputs(rows, V, k, "f32", 4)
    x[0, idx[0, 0]] = -math.inf
    w[0] = 1.0
    loss, _, _, grad, _ = _check(x, idx, logp, w, 1.0, True)
    assert loss[0] == math.inf and abs(grad[0, idx[0, 0]].item() + math.exp(logp[0, 0].item())) < 1e-6
    # broken rows stay in their places
    x[1, 7], x[2, 9] = math.nan, math.inf
    loss = Q.qadc_distill(x, idx, logp)[0]
    step_loss, step = Q.qadc_distill_step(x, idx, logp, torch.ones_like(w))
    assert torch.isnan(loss[1:3]).all() and torch.isnan(step_loss[1:3]).all() and torch.isnan(step[1:3]).all()
    assert torch.isfinite(loss[3:]).all() and torch.isfinite(step[3:]).all()
    # rows without a share of the loss: zeros, whatever they hold
    none = torch.zeros_like(w)
    assert (Q.qadc_distill_step(x, idx, logp, none)[1] == 0).all()
    assert (Q.qadc_distill_backward(x, idx, logp, loss, loss, none) == 0).all()


@pytest.mark.parametrize("rows,V", [(5, 500), (200, 500), (5, 50021), (130, 70001), (410, 41000)])
def test_rows_of_nothing_but_nan(rows, V):
    """A NaN with nothing beside it, stored or not, is no row with nothing left."""
    import paper_1704_07355_amd as Q
    for type in TYPES:
        x, idx, logp, w = _inputs(rows, V, 12, type, 5)
        w = w.abs() + 0.1
        x[:4] = -math.inf
        x[0] = math.nan
        x[1, 450] = math.nan
        idx[1] = torch.arange(12, device=DEV)
        x[2, idx[2, 0]] = math.nan
        for tail in (True, False):
            loss, lse, log_tail = Q.qadc_distill(x, idx, logp, 1.0, tail)
            step_loss, step = Q.qadc_distill_step(x, idx, logp, w, 1.0, tail)
            grad = Q.qadc_distill_backward(x, idx, logp, lse, log_tail, w, 1.0, tail)
            for t in (loss, lse, step_loss, step.float(), grad.float()):
                assert torch.isnan(t[:3]).all() and not torch.isnan(t[3:]).any()
            assert loss[3] == step_loss[3] == math.inf and lse[3] == log_tail[3] == -math.inf
            assert (step[3] == 0).all() and (grad[3] == 0).all()


@pytest.mark.parametrize("rows", [4, 160])
def test_a_student_that_gives_the_tail_next_to_nothing(rows):
    """Q down to 1e-25 keeps its gradient, whatever the row's share of the loss; below 2^-100 it counts as nothing."""
    import paper_1704_07355_amd as Q
    V, k = 400, 12
    g = gen(21)
    idx = torch.stack([torch.randperm(V, generator=g, device=DEV)[:k] for _ in range(rows)]).to(torch.int32)
    logp = torch.log_softmax(torch.randn((rows, k), generator=g, device=DEV), 1) - 0.5
    for depth in (20.0, 45.0, 60.0):
        x = torch.randn((rows, V), generator=g, device=DEV) - depth
        x.scatter_(1, idx.long(), torch.randn((rows, k), generator=g, device=DEV))
        _check(x, idx, logp, 100.0 * torch.rand((rows,), generator=g, device=DEV), 1.0, True)
    x -= 30.0 * (x < -20.0)
    w = torch.ones((rows,), device=DEV)
    loss, lse, log_tail = Q.qadc_distill(x, idx, logp)
    grad = Q.qadc_distill_backward(x, idx, logp, lse, log_tail, w)
    step_loss, step = Q.qadc_distill_step(x, idx, logp, w)
    assert (log_tail == -math.inf).all() and torch.isfinite(loss).all() and torch.isfinite(step_loss).all()
    others = torch.ones((rows, V), dtype=torch.bool, device=DEV).scatter_(1, idx.long(), False)
    assert grad[others].abs().max() < 2.0 ** -99 and step[others].abs().max() < 2.0 ** -99


@pytest.mark.parametrize("rows,V", [(6, 500), (200, 500), (6, 50021), (130, 70001)])
def test_broken_rows_of_an_empty_teacher(rows, V):
    """A NaN or an infinity shows in the loss as it does in the gradient, whatever the teacher says; without one an empty teacher has none."""
    import paper_1704_07355_amd as Q
    for type in TYPES:
        x, idx, logp, w = _inputs(rows, V, 12, type, 5)
        w = w.abs() + 0.1
        idx[:4] = -1
        x[0, V - 1], x[1, V // 2], x[2] = math.nan, math.inf, -math.inf
        x[4, 7] = math.nan
        for tail in (True, False):
            for teacher in ((idx, logp), (idx[:, :0].contiguous(), logp[:, :0].contiguous())):
                loss, lse, log_tail = Q.qadc_distill(x, *teacher, 1.0, tail)
                step_loss, step = Q.qadc_distill_step(x, *teacher, w, 1.0, tail)
                grad = Q.qadc_distill_backward(x, *teacher, lse, log_tail, w, 1.0, tail)
                for t in (loss, step_loss, step.float(), grad.float()):
                    assert torch.isnan(t[[0, 1, 4]]).all() and not torch.isnan(t[[2, 3, 5]]).any()
                assert loss[2] == step_loss[2] == 0 and (step[2] == 0).all() and (grad[2] == 0).all()
                if not tail:
                    assert loss[3] == step_loss[3] == 0 and (step[3] == 0).all() and (grad[3] == 0).all()


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("rows,V,k", [(4, 400, 12), (160, 400, 12), (3, 7001, 128), (70, 60001, 20), (90, 131072, 40), (2, 140001, 9)])
def test_a_tail_of_any_depth_counts(rows, V, k, type):
    """Q between 1e-24 and 1e-36 has its term in the loss and its gradient, in one call and in two, also where no single token's share
    is a float32 any more; the log probabilities of the tokens beside it are those of the definition."""
    g = gen(V)
    idx = torch.stack([torch.randperm(V, generator=g, device=DEV)[:k] for _ in range(rows)]).to(torch.int32)
    logp = torch.log_softmax(torch.randn((rows, k), generator=g, device=DEV), 1) - 0.5
    w = 0.1 + torch.rand((rows,), generator=g, device=DEV)
    for share in (1e-24, 1e-29, 1e-31, 1e-34, 1e-36):
        # (the logits' mean exponential is exp(1/2) of that of their mean, among the stored tokens and the others)
        depth = math.log(V / k / share)
        x = torch.randn((rows, V), generator=g, device=DEV) - depth
        x.scatter_(1, idx.long(), torch.randn((rows, k), generator=g, device=DEV))
        loss, lse, log_tail, grad, step = _check(x.to(TYPES[type]), idx, logp, w, 1.0, True)
        assert torch.isfinite(log_tail).all() and (loss > 8.0).all()  # r (log r - log Q), r = 0.39, of which is 21 to 33
        # a scale between the logits and their exponentials moves nothing
        _check((2.0 * x).to(TYPES[type]), idx, logp, w, 0.5, True)


@pytest.mark.parametrize("rows", [3, 150])
def test_gradient_against_differences(rows):
    """Central differences of sum(w loss) in 64 bits, along random directions."""
    import paper_1704_07355_amd as Q
    V, k = 300, 10
    x, idx, logp, w = _inputs(rows, V, k, "f32", 12, scale=0.8)
    for tail in (True, False):
        step = Q.qadc_distill_step(x, idx, logp, w, 0.8, tail)[1].double()
        ref = _reference(x, idx, logp, 0.8, tail)
        want, lp, q, share, ratio, f = _gradient(ref, ref["lse"], ref["log_tail"], w, 0.8)
        E = 4 * _error(V)
        for seed in range(3):
            u = torch.randn((rows, V), generator=gen(seed), device=DEV).double()
            t = 1e-4
            ends = []
            for sign in (1, -1):
                y = x.double() + sign * t * u
                ends.append((w.double() * _reference(y, idx, logp, 0.8, tail)["loss"]).sum())
            slope = (ends[0] - ends[1]) / (2 * t)
            size = f * ((share.abs() + ratio) * q * ((2 * lp.abs() + 8) * EPS + E) + 6 * EPS * ref["p"])
            tol = (size * u.abs()).sum() + t * t * (f * (u.abs() ** 3) * (q + ref["p"]) * 10).sum()
            assert abs(((step * u).sum() - slope).item()) <= tol.item()


def test_the_alternatives_of_a_teacher_are_what_is_stored():
    """A student that is the teacher has no loss and no gradient; the alternatives go in as they come out, padded too."""
    import paper_1704_07355_amd as Q
    for rows, V, k in ((4, 20000, 50), (200, 900, 20), (3, 5, 9)):
        x = 2.0 * torch.randn((rows, V), generator=gen(V), device=DEV)
        top, top_logp = Q.qadc_token_logprobs(x, k=k, scale=0.7)[3:5]
        E = _error(V)
        loss, lse, log_tail = Q.qadc_distill(x, top, top_logp, 0.7)
        assert loss.abs().max().item() <= 8 * E + 40 * EPS
        g = Q.qadc_distill_step(x, top, top_logp, torch.ones(rows, device=DEV), 0.7)[1]
        assert g.abs().max().item() <= 8 * E + 40 * EPS


@pytest.mark.parametrize("V", [20000, 50000])
def test_equal_calls_give_equal_bits_and_a_workspace_serves_fewer_rows(V):
    import paper_1704_07355_amd as Q
    x, idx, logp, w = _inputs(420, V, 20, "bf16", 3)
    ws = torch.empty(Q.qadc_distill_workspace_bytes(420, V), dtype=torch.uint8, device=DEV)
    for rows in (1, 2, 7, 64, 127, 128, 399, 400, 420):
        a = Q.qadc_distill_step(x[:rows], idx[:rows], logp[:rows], w[:rows], workspace=ws)
        b = Q.qadc_distill(x[:rows], idx[:rows], logp[:rows], workspace=ws)
        ws.fill_(255)
        c = Q.qadc_distill_step(x[:rows], idx[:rows], logp[:rows], w[:rows], workspace=ws)
        d = Q.qadc_distill(x[:rows], idx[:rows], logp[:rows], workspace=ws)
        assert all(torch.equal(p, q) for p, q in zip(a + b, c + d))
    for V in (1, 8192, 20000, 300000):
        most = Q.qadc_distill_workspace_bytes(1000, V)
        assert all(Q.qadc_distill_workspace_bytes(r, V) <= most for r in (1, 2, 100, 399, 400, 401, 999))


def test_a_large_gradient_is_that_of_its_rows():
    """Beyond the last cache's size the stores go past it; the bits stay."""
    import paper_1704_07355_amd as Q
    rows, V, k = 3300, 64001, 20
    x = torch.randn((rows, V), generator=gen(7), device=DEV, dtype=torch.bfloat16)
    _, idx, logp, w = _inputs(rows, 200, k, "bf16", 8)
    lse, log_tail = Q.qadc_distill(x, idx, logp)[1:]
    room = apart(torch.zeros_like(x), V + 5, 3)
    Q.qadc_distill_backward(x, idx, logp, lse, log_tail, w, out=room)
    for r in range(0, rows, 1100):
        part = slice(r, r + 1100)
        want = Q.qadc_distill_backward(x[part], idx[part], logp[part], lse[part], log_tail[part], w[part])
        assert torch.equal(room[part], want)
    assert torch.isnan(torch.as_strided(room, (rows - 1, 5), (V + 5, 1), room.storage_offset() + V).float()).all()


def test_no_rows_and_wrong_tensors():
    import paper_1704_07355_amd as Q
    x, idx, logp, w = _inputs(4, 100, 5, "f16", 3)
    assert Q.qadc_distill_step(x[:0], idx[:0], logp[:0], w[:0])[1].shape == (0, 100)
    assert Q.qadc_distill(x[:0], idx[:0], logp[:0])[0].numel() == 0
    lse = torch.zeros_like(w)
    for call in (lambda: Q.qadc_distill(x, idx[:3], logp[:3]), lambda: Q.qadc_distill(x, idx, logp[:, :4]), lambda: Q.qadc_distill(x, idx.long(), logp),
                 lambda: Q.qadc_distill(x, idx, logp.double()), lambda: Q.qadc_distill(x.double(), idx, logp),
                 lambda: Q.qadc_distill_step(x, idx, logp, w[:3]), lambda: Q.qadc_distill_step(x, idx, logp, w, out=x[:3]),
                 lambda: Q.qadc_distill_backward(x, idx, logp, lse, lse[:3], w),
                 lambda: Q.qadc_distill_backward(x, idx, logp, lse, lse, w, out=x.float())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: Q.qadc_distill(x, idx, logp, -1.0), lambda: Q.qadc_distill_step(x, idx, logp, w, workspace=torch.empty(256, dtype=torch.uint8, device=DEV))):
        with pytest.raises(Q.QadcError):
            call()
