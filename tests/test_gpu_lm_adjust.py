"""Penalties, biases and masks on logits against their definition in 64 bits.

Tolerances, from the arithmetic (u: half a unit in the last place of the output's type, e = 2^-24): an adjusted logit is a
quotient or product, a product and two sums, and a sum of b biases: at most 4 + b roundings to float32 of numbers that are at most
the sum of the magnitudes, then one to the output's type.  All other logits are equal bit by bit.
"""

import math

import numpy as np
import pytest

import torch

from lm_common import DEV, EPS, LEAST, TYPES, UNIT, apart, gen, within

pytestmark = pytest.mark.gpu


def _bits(t):
    return t.view(torch.int32 if t.element_size() == 4 else torch.int16)


def _pack(allowed):
    """Masks [states][V] of truth values as words, with bits behind the last token set at random."""
    a = allowed.cpu().numpy()
    states, V = a.shape
    words = -(-V // 32)
    full = np.ones((states, words * 32), dtype=bool)
    full[:, :V] = a
    return torch.from_numpy(np.packbits(full, axis=1, bitorder="little").view(np.int32).copy()).to(DEV)


def _want(x, kw, V):
    """The definition, row by row in 64 bits -> (values, magnitudes that were added, roundings, touched)."""
    rows = x.shape[0]
    out, size, count = x.double().clone(), x.double().abs(), torch.zeros(x.shape, dtype=torch.float64, device=DEV)
    touched = torch.zeros(x.shape, dtype=torch.bool, device=DEV)
    for r in range(rows):
        if kw.get("history") is not None:
            h = kw["history"][r]
            n = h.numel() if kw.get("lengths") is None else min(max(int(kw["lengths"][r]), 0), h.numel())
            m = 0 if kw.get("prompt") is None else max(int(kw["prompt"][r]), 0)

            def times(part):
                part = part[(part >= 0) & (part < V)].long()
                return torch.bincount(part, minlength=V).double()

            seen, said = times(h[:n]) > 0, times(h[min(m, n):n])
            rep, pres, freq = (float(kw[k][r]) if kw.get(k) is not None else d
                               for k, d in (("repetition", 1.0), ("presence", 0.0), ("frequency", 0.0)))
            y = torch.where(out[r] > 0, out[r] / rep, out[r] * rep)
            out[r] = torch.where(seen, y, out[r])
            off = freq * said + pres * (said > 0)
            out[r] = torch.where(said > 0, out[r] - off, out[r])
            size[r] = torch.where(seen, y.abs(), size[r]) + freq * said + abs(pres)
            touched[r] |= seen
        if kw.get("bias") is not None:
            t, b = kw["bias_tokens"][r].long(), kw["bias"][r].double()
            some = (t >= 0) & (t < V)
            out[r].index_add_(0, t[some], b[some])
            size[r].index_add_(0, t[some], b[some].abs())
            count[r].index_add_(0, t[some], torch.ones_like(b[some]))
            touched[r, t[some]] = True
        if kw.get("allowed") is not None:
            s = r if kw.get("mask_of") is None else int(kw["mask_of"][r])
            if 0 <= s < kw["allowed"].shape[0]:
                out[r][~kw["allowed"][s]] = -math.inf
                touched[r] |= ~kw["allowed"][s]
    return out, size, count, touched


def _check(x, kw, **how):
    import paper_1704_07355_amd as Q
    type = [k for k, t in TYPES.items() if t == x.dtype][0]
    before = x.clone()
    args = {k: v for k, v in kw.items() if k != "allowed"}
    got = Q.qadc_adjust_logits(x, **args, **how)
    want, size, count, touched = _want(before, kw, x.shape[1])
    assert got.dtype == x.dtype and torch.equal(_bits(got.contiguous())[~touched], _bits(before.contiguous())[~touched])
    within(got, want, UNIT[type] * want.abs() + LEAST[type] + (4 + count) * EPS * size * (1 + UNIT[type]), "adjusted")
    if how.get("out") is not x:
        assert torch.equal(_bits(x.contiguous()), _bits(before.contiguous()))
    return got


def _rules(rows, V, H, B, masked, seed, unused=True):
    g = gen(seed)
    kw = {}
    rand = lambda *s: torch.rand(s, generator=g, device=DEV)
    if H:
        kw["history"] = (rand(rows, H) ** 3 * V).to(torch.int32).clamp_(max=V - 1)
        if unused:
            kw["history"][rand(rows, H) < 0.1] = -1
            kw["history"][rand(rows, H) < 0.05] = V
        kw["lengths"] = (rand(rows) * (H + 1)).to(torch.int32)
        kw["lengths"][0] = H
        kw["lengths"][rows // 2] = 0 if rows > 1 else H
        kw["prompt"] = (kw["lengths"] * rand(rows)).to(torch.int32)
        kw["repetition"], kw["presence"], kw["frequency"] = 0.7 + rand(rows), rand(rows) - 0.3, 0.4 * rand(rows)
    if B:
        kw["bias_tokens"] = (rand(rows, B) * V).to(torch.int32).clamp_(max=V - 1)
        if unused:
            kw["bias_tokens"][rand(rows, B) < 0.2] = -1
        kw["bias"] = 4.0 * rand(rows, B) - 2.0
    if masked:
        states = 3
        kw["allowed"] = rand(states, V) < torch.tensor([[0.6], [0.02], [0.0]], device=DEV)  # the last leaves nothing
        kw["masks"] = _pack(kw["allowed"])
        kw["mask_of"] = torch.randint(-1, states + 1, (rows,), generator=g, device=DEV, dtype=torch.int32)
    return kw


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("rows,V,H,B,masked", [
    (1, 1, 1, 1, True), (3, 7, 20, 5, True), (2, 31, 4, 0, False), (2, 33, 0, 9, True), (5, 1000, 1023, 64, True),
    (4, 2047, 5, 3, False), (4, 2048, 1024, 0, True), (4, 2049, 1025, 1, True), (3, 5003, 4099, 200, True), (2, 20001, 9000, 1024, False),
    (1, 131072, 2048, 16, True), (70, 1024, 100, 10, True), (2, 70001, 40000, 7, True), (9, 1023, 0, 0, True), (9, 1025, 3, 0, False)])
def test_rules(rows, V, H, B, masked, type):
    x = (3.0 * torch.randn((rows, V), generator=gen(V + H), device=DEV)).to(TYPES[type])
    kw = _rules(rows, V, H, B, masked, 3 * V + H)
    got = _check(x, kw)
    again = x.clone()
    assert torch.equal(_bits(_check(again, kw, out=again)), _bits(got))  # in place


@pytest.mark.parametrize("type", list(TYPES))
def test_each_rule_alone(type):
    rows, V = 6, 3001
    x = (3.0 * torch.randn((rows, V), generator=gen(2), device=DEV)).to(TYPES[type])
    all = _rules(rows, V, 700, 40, True, 5)
    h = {"history": all["history"]}
    for kw in ({}, h, dict(h, lengths=all["lengths"]), dict(h, repetition=all["repetition"]), dict(h, presence=all["presence"]),
               dict(h, frequency=all["frequency"]), dict(h, frequency=all["frequency"], prompt=all["prompt"]),
               {k: all[k] for k in ("bias", "bias_tokens")}, {k: all[k] for k in ("allowed", "masks", "mask_of")}):
        _check(x, kw)
    # a mask for every row, in order
    allowed = torch.rand((rows + 1, V), generator=gen(8), device=DEV) < 0.5
    _check(x, {"allowed": allowed, "masks": _pack(allowed)})


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("V,ld,shift", [(1000, 1003, 1), (2051, 4000, 3), (9, 9, 5), (300, 301, 7)])
def test_rows_apart_and_unaligned(V, ld, shift, type):
    import paper_1704_07355_amd as Q
    rows = 5
    x = (3.0 * torch.randn((rows, V), generator=gen(V), device=DEV)).to(TYPES[type])
    kw = _rules(rows, V, 333, 20, True, V)
    args = {k: v for k, v in kw.items() if k != "allowed"}
    want = Q.qadc_adjust_logits(x, **args)
    wide = apart(x, ld, shift)
    room = apart(x, ld + 3, shift + 1)
    args["masks"] = apart(kw["masks"].view(torch.float32), kw["masks"].shape[1] + 3, 1).view(torch.int32)
    assert torch.equal(_bits(Q.qadc_adjust_logits(wide, **args, out=room).contiguous()), _bits(want))
    if ld > V:
        assert torch.isnan(torch.as_strided(room, (rows - 1, 3), (ld + 3, 1), room.storage_offset() + V).float()).all()
    assert torch.equal(_bits(Q.qadc_adjust_logits(wide, **args, out=wide).contiguous()), _bits(want))


def test_same_token_many_times_adds_in_order():
    """Repeated biases are added in the order in which they are given, counts are whole numbers: equal calls give equal bits."""
    import paper_1704_07355_amd as Q
    rows, V, B = 4, 4000, 1024
    g = gen(6)
    x = torch.randn((rows, V), generator=g, device=DEV)
    tokens = torch.randint(0, 50, (rows, B), generator=g, device=DEV, dtype=torch.int32) * 80
    bias = torch.randn((rows, B), generator=g, device=DEV) * 10.0 ** torch.randint(-3, 4, (rows, B), generator=g, device=DEV)
    got = Q.qadc_adjust_logits(x, bias_tokens=tokens, bias=bias)
    sums = torch.zeros((rows, V), device="cpu")
    for r in range(rows):
        for t, b in zip(tokens[r].tolist(), bias[r].cpu()):
            sums[r, t] += b  # one float32 addition after the other
    assert torch.equal(got.cpu(), torch.where(sums != 0, x.cpu() + sums, x.cpu()))
    # one token 50000 times
    h = torch.full((rows, 50000), 123, device=DEV, dtype=torch.int32)
    y = Q.qadc_adjust_logits(x, h, frequency=torch.full((rows,), 0.25, device=DEV))
    assert torch.equal(y[:, 123].double(), (x[:, 123].double() - 12500.0).float().double())
    assert torch.equal(y[:, 122], x[:, 122])


def test_infinities_and_nan():
    import paper_1704_07355_amd as Q
    x = torch.tensor([[math.inf, -math.inf, math.nan, 1.0, -2.0, math.inf, math.nan, -math.inf]], device=DEV)
    h = torch.tensor([[0, 1, 2, 4, 7]], device=DEV, dtype=torch.int32)
    two = torch.full((1,), 2.0, device=DEV)
    allowed = torch.ones((1, 8), dtype=torch.bool, device=DEV)
    allowed[0, 5:7] = False
    y = Q.qadc_adjust_logits(x, h, repetition=two, frequency=two, masks=_pack(allowed),
                             bias_tokens=torch.tensor([[3]], device=DEV, dtype=torch.int32), bias=torch.tensor([[-math.inf]], device=DEV))[0].tolist()
    assert y[0] == math.inf and y[1] == -math.inf and math.isnan(y[2]) and y[3] == -math.inf and y[4] == -6.0
    assert y[5] == y[6] == y[7] == -math.inf
    # the result feeds the log probabilities: a row with nothing left
    z = Q.qadc_adjust_logits(x, masks=_pack(torch.zeros((1, 8), dtype=torch.bool, device=DEV)))
    lse, top = Q.qadc_token_logprobs(z, k=3)[1], Q.qadc_token_logprobs(z, k=3)[4]
    assert lse.item() == -math.inf and (top == -math.inf).all()


def test_no_rows_and_wrong_tensors():
    import paper_1704_07355_amd as Q
    x = torch.randn((3, 100), device=DEV)
    assert Q.qadc_adjust_logits(x[:0]).shape == (0, 100)
    h = torch.zeros((3, 5), dtype=torch.int32, device=DEV)
    one = torch.ones((3,), device=DEV)
    masks = torch.zeros((3, 4), dtype=torch.int32, device=DEV)
    for call in (lambda: Q.qadc_adjust_logits(x, h[:2]), lambda: Q.qadc_adjust_logits(x, h.long()), lambda: Q.qadc_adjust_logits(x, presence=one),
                 lambda: Q.qadc_adjust_logits(x, h, presence=one[:2]), lambda: Q.qadc_adjust_logits(x, h, presence=one.double()),
                 lambda: Q.qadc_adjust_logits(x, bias_tokens=h), lambda: Q.qadc_adjust_logits(x, bias_tokens=h, bias=one),
                 lambda: Q.qadc_adjust_logits(x, masks=masks[:, :3]), lambda: Q.qadc_adjust_logits(x, masks=masks.long()),
                 lambda: Q.qadc_adjust_logits(x, mask_of=h[:, 0]), lambda: Q.qadc_adjust_logits(x.double()),
                 lambda: Q.qadc_adjust_logits(x, out=x[:2]), lambda: Q.qadc_adjust_logits(x, out=x.half())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(Q.QadcError):
        Q.qadc_adjust_logits(x, masks=masks[:2])  # fewer masks than rows
