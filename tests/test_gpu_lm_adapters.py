"""Low-rank adapters of many requests against their formula in 64 bits.

Tolerances, from the arithmetic (v: half a unit in the last place of the type, e = 2^-24): u = A x has chains of at most K/4 + 40
float32 additions, each off by e of the magnitudes summed so far (a float32 product one more); between the products u keeps 2^-16 (bfloat16) or
2^-22 and 2^-35 of its row's largest (binary16); the second sum has chains of at most 2 rank + 8, and the addition of base and the rounding to
the type follow.
"""

import math

import pytest

import torch

from lm_common import DEV, EPS, LEAST, TYPES, UNIT, apart, gen, within

pytestmark = pytest.mark.gpu

KEPT = {"f32": 0.0, "f16": 2.0 ** -22, "bf16": 2.0 ** -16}


def _pool(count, rank, N, K, type, seed, ranks=True, scales=True):
    """A pool whose unused ranks hold NaN."""
    import paper_1704_07355_amd as Q
    g = gen(seed)
    t = TYPES[type]
    a = (torch.randn((count, rank, K), generator=g, device=DEV) / math.sqrt(K)).to(t)
    b = torch.randn((count, N, rank), generator=g, device=DEV).to(t)
    r = s = None
    if ranks:
        r = torch.randint(0, rank + 1, (count,), generator=g, device=DEV, dtype=torch.int32)
        r[0], r[-1] = rank, max(1, rank // 2)
        unused = torch.arange(rank, device=DEV)[None, :] >= r[:, None]
        a.masked_fill_(unused[:, :, None], math.nan)
        b.masked_fill_(unused[:, None, :], math.nan)
    if scales:
        s = 2.0 * torch.rand((count,), generator=g, device=DEV) - 0.5
    return Q.qadc_adapters(a, b, s, r)


def _rows(M, N, K, type, seed):
    g = gen(seed)
    x = (torch.randn((M, K), generator=g, device=DEV) * (0.2 + 3.0 * torch.rand((M, 1), generator=g, device=DEV))).to(TYPES[type])
    return x, torch.randn((M, N), generator=g, device=DEV).to(TYPES[type])


def _want(w, ids, x, base, type):
    a, b, scales, ranks = w.tensors
    want = torch.zeros((x.shape[0], w.N), dtype=torch.float64, device=DEV) if base is None else base.double().clone()
    err = torch.zeros_like(want)
    x64 = x.double()
    for i in ids.unique().tolist():
        if not 0 <= i < w.count:
            continue
        at = (ids == i).nonzero()[:, 0]
        r = w.rank if ranks is None else min(max(int(ranks[i]), 0), w.rank)
        if r == 0:
            continue
        s = 1.0 if scales is None else float(scales[i])
        A, B = a[i, :r].double().t().contiguous(), b[i, :, :r].double().t().contiguous()
        u = torch.mm(x64[at], A)
        du = (w.K / 4 + 42) * EPS * torch.mm(x64[at].abs(), A.abs()) + (KEPT[type] + 2 * EPS) * u.abs()
        if type == "f16":
            du = du + 2.0 ** -35 * u.abs().amax(1, keepdim=True)
        delta, size = torch.mm(u, B) * s, torch.mm(u.abs(), B.abs()) * abs(s)
        want[at] += delta
        err[at] += torch.mm(du, B.abs()) * abs(s) + (2 * w.rank + 10) * EPS * size
    total = want.abs() + err
    return want, UNIT[type] * total + LEAST[type] + err + 2 * EPS * (total + (0.0 if base is None else base.double().abs()))


def _check(w, ids, x, base, **how):
    import paper_1704_07355_amd as Q
    type = [k for k, t in TYPES.items() if t == x.dtype][0]
    before = None if base is None else base.clone()
    want, tol = _want(w, ids, x, before, type)
    y = Q.qadc_add_adapters(w, ids, x, base, **how)
    within(y, want, tol, "y")
    none = (ids < 0) | (ids >= w.count)
    if before is not None:
        assert torch.equal(y[none], before[none])
    return y


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("M,N,K,rank,count", [(1, 1, 1, 1, 1), (1, 64, 64, 16, 3), (2, 65, 33, 8, 2), (5, 257, 100, 3, 4), (16, 100, 1000, 17, 5),
                                              (17, 300, 4096, 64, 9), (64, 1000, 515, 16, 40), (255, 70, 96, 33, 300), (257, 130, 130, 128, 7),
                                              (700, 513, 260, 100, 3), (64, 2000, 31, 5, 1), (3, 5000, 3000, 16, 2), (1000, 40, 2000, 20, 2),
                                              (1100, 333, 520, 64, 11), (1030, 130, 2100, 128, 16), (1500, 50, 200, 40, 23),
                                              (1200, 300, 64, 5, 3), (1024, 200, 640, 128, 1)])
def test_mixed_rows(M, N, K, rank, count, type):
    w = _pool(count, rank, N, K, type, M + N)
    x, base = _rows(M, N, K, type, K)
    ids = torch.randint(-1, count + 1, (M,), generator=gen(M), device=DEV, dtype=torch.int32)
    ids[0] = 0
    y = _check(w, ids, x, base)
    _check(w, ids, x, None)
    again = base.clone()
    assert torch.equal(_check(w, ids, x, again, out=again), y)  # in place


def test_more_outputs_than_a_launch_has_workgroups_for(memory_back):
    """256 rows, each of which may open an item, by 2^27 outputs and some: the pool repeats itself, and so has the result to."""
    import paper_1704_07355_amd as Q
    M, N, K, rank, count, period = 256, (1 << 27) + 4096, 40, 8, 4, 4096
    small = _pool(count, rank, period, K, "bf16", 3)
    a, b, scales, ranks = small.tensors
    w = Q.qadc_adapters(a, b.repeat(1, N // period, 1), scales, ranks)
    x, _ = _rows(M, period, K, "bf16", 3)
    ids = torch.randint(-1, count + 1, (M,), generator=gen(1), device=DEV, dtype=torch.int32)
    y = Q.qadc_add_adapters(w, ids, x)
    want, tol = _want(small, ids, x, None, "bf16")
    within(y[:, :period], want, tol, "y")
    for r in range(M):
        row = y[r].view(-1, period)
        same = torch.equal(row, row[:1].expand(row.shape))
        assert same, r


def test_more_rows_than_tiles_with_a_workgroup_for_each_row():
    w = _pool(1100, 8, 64, 24, "bf16", 5)
    x, base = _rows(70001, 64, 24, "bf16", 5)
    _check(w, torch.randint(-1, 1101, (70001,), generator=gen(6), device=DEV, dtype=torch.int32), x, base)


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("M,count", [(256, 1), (300, 4), (1000, 3), (513, 2), (640, 10), (1100, 3), (2000, 7)])
def test_segments(M, count, type):
    """Requests one after the other, of lengths that end inside tiles, one of them without an adapter."""
    import paper_1704_07355_amd as Q
    for rank, ranks, scales in ((16, False, False), (64, True, True), (40, True, False)):
        w = _pool(count, rank, 333, 520, type, rank, ranks, scales)
        x, base = _rows(M, 333, 520, type, M)
        cut = torch.sort(torch.randint(0, M, (count,), generator=gen(count), device=DEV)).values
        ids = (torch.searchsorted(cut, torch.arange(M, device=DEV), right=True) - 1).to(torch.int32)
        _check(w, ids, x, base)
        # a row's result does not depend on where it lies or on what lies beside it, but for the cuts of the inputs
        turn = torch.randperm(M, generator=gen(1), device=DEV)
        mixed = Q.qadc_add_adapters(w, ids[turn].contiguous(), x[turn].contiguous(), base[turn].contiguous())
        assert torch.equal(mixed, Q.qadc_add_adapters(w, ids, x, base)[turn])


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("M", [6, 300])
def test_rows_apart_and_unaligned(M, type):
    import paper_1704_07355_amd as Q
    N, K = 201, 77
    w = _pool(3, 9, N, K, type, 4)
    x, base = _rows(M, N, K, type, 4)
    ids = torch.arange(M, device=DEV, dtype=torch.int32) % 4
    want = _check(w, ids, x, base)
    room = apart(base, N + 5, 1)
    got = Q.qadc_add_adapters(w, ids, apart(x, K + 3, 1), apart(base, N + 2, 3), out=room)
    assert torch.equal(got, want)
    assert torch.isnan(torch.as_strided(room, (M - 1, 5), (N + 5, 1), room.storage_offset() + N).float()).all()
    inside = apart(base, N + 1, 1)
    assert torch.equal(Q.qadc_add_adapters(w, ids, x, inside, out=inside), want)


@pytest.mark.parametrize("type", list(TYPES))
def test_broken_rows_stay_in_their_places(type):
    import paper_1704_07355_amd as Q
    for M in (20, 400):
        w = _pool(2, 16, 150, 200, type, 8, False)
        x, base = _rows(M, 150, 200, type, 8)
        ids = torch.arange(M, device=DEV, dtype=torch.int32) % 3
        want = Q.qadc_add_adapters(w, ids, x, base)
        x[3, 7], x[6, 9] = math.nan, math.inf
        base[10, 11] = math.nan
        got = Q.qadc_add_adapters(w, ids, x, base)
        broken = torch.tensor([3, 6, 10], device=DEV)
        rest = torch.ones(M, dtype=torch.bool, device=DEV)
        rest[broken] = False
        assert torch.equal(got[rest], want[rest])
        assert not torch.isfinite(got[3]).any() and not torch.isfinite(got[6]).any()
        assert torch.isnan(got[10]).sum() == 1


def test_large_and_small_values_between_the_products():
    """Binary16: u far beyond its range, and far below it, with a pool whose products come back."""
    import paper_1704_07355_amd as Q
    K, N = 256, 64
    for size in (2.0 ** 9, 2.0 ** -12):
        a = torch.full((1, 1, K), size, device=DEV).half()
        x = torch.full((3, K), size, device=DEV).half()
        b = torch.full((1, N, 1), 2.0 ** -14 if size > 1 else 2.0 ** 14, device=DEV).half()
        w = Q.qadc_adapters(a, b)
        y = Q.qadc_add_adapters(w, torch.zeros(3, dtype=torch.int32, device=DEV), x)
        assert torch.equal(y.double(), torch.full((3, N), K * size * size * float(b[0, 0, 0]), dtype=torch.float64, device=DEV).half().double())


def test_beside_the_shared_projection():
    """A product with 4-bit weights and the adapters of its rows, as they are used together."""
    import paper_1704_07355_amd as Q
    M, N, K = 12, 300, 256
    g = gen(2)
    codes = torch.randint(0, 256, (N, K // 2), generator=g, device=DEV, dtype=torch.uint8)
    scales = (0.02 * torch.rand((N, K // 128), generator=g, device=DEV)).to(torch.bfloat16)
    shared = Q.qadc_pack_weights4(codes, scales, None, K, 128)
    w = _pool(4, 8, N, K, "bf16", 5)
    x, _ = _rows(M, N, K, "bf16", 6)
    ids = torch.arange(M, device=DEV, dtype=torch.int32) % 5
    y = Q.qadc_linear4(shared, x)
    _check(w, ids, x, y.clone(), out=y.clone())
    want = Q.qadc_add_adapters(w, ids, x, y)
    assert torch.equal(Q.qadc_add_adapters(w, ids, x, y, out=y), want)


def test_equal_calls_give_equal_bits_and_a_workspace_serves_fewer_rows():
    import paper_1704_07355_amd as Q
    w = _pool(30, 16, 500, 3000, "bf16", 3)
    x, base = _rows(600, 500, 3000, "bf16", 3)
    ids = torch.randint(-1, 30, (600,), generator=gen(5), device=DEV, dtype=torch.int32)
    ws = torch.empty(Q.qadc_adapters_workspace_bytes(w, 600), dtype=torch.uint8, device=DEV)
    for M in (1, 2, 15, 16, 17, 64, 255, 256, 257, 600):
        a = Q.qadc_add_adapters(w, ids[:M], x[:M], base[:M], workspace=ws)
        ws.fill_(255)
        assert torch.equal(a, Q.qadc_add_adapters(w, ids[:M], x[:M], base[:M], workspace=ws))


def test_no_rows_and_wrong_tensors():
    import paper_1704_07355_amd as Q
    w = _pool(3, 8, 50, 40, "f16", 3)
    x, base = _rows(4, 50, 40, "f16", 3)
    ids = torch.zeros(4, dtype=torch.int32, device=DEV)
    assert Q.qadc_add_adapters(w, ids[:0], x[:0], base[:0]).shape == (0, 50)
    a, b = w.tensors[:2]
    for call in (lambda: Q.qadc_add_adapters(w, ids[:3], x, base), lambda: Q.qadc_add_adapters(w, ids.long(), x, base),
                 lambda: Q.qadc_add_adapters(w, ids, x[:, :39], base), lambda: Q.qadc_add_adapters(w, ids, x.float(), base),
                 lambda: Q.qadc_add_adapters(w, ids, x, base[:3]), lambda: Q.qadc_add_adapters(w, ids, x, base, out=base[:, :49]),
                 lambda: Q.qadc_adapters(a, b[:, :, :7]), lambda: Q.qadc_adapters(a, b.float()), lambda: Q.qadc_adapters(a[0], b[0]),
                 lambda: Q.qadc_adapters(a, b, torch.ones(2, device=DEV)), lambda: Q.qadc_adapters(a.transpose(1, 2), b)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(Q.QadcError):
        Q.qadc_add_adapters(w, ids, x, base, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
