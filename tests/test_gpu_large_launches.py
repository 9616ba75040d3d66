"""Database-side calls of so many vectors, codes or cells that a launch of a thread for each passes 32 bits: what lies at the end is computed
too.  The same rows in a small call are the reference (which other tests compare with the oracle)."""

import pytest

import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
MANY = 1 << 32


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _places(n, width=1000):
    """Stretches of a list of n: its beginning, across 2^31 and 2^32 and their halves, its end."""
    return [slice(max(0, at - width), min(n, at + width)) for at in (0, n // 2, 1 << 30, 1 << 31, MANY, n) if at <= n]


def test_codes_of_many_vectors(memory_back):
    import paper_1704_07355_amd as Q
    n = MANY + 77
    codebooks = torch.randn((2, 256, 1), generator=_gen(1), device=DEV)
    x = torch.empty((n, 2), device=DEV)
    for part in x.split(1 << 28):
        part.normal_(generator=_gen(2))
    codes = Q.qadc_pq_encode(codebooks, x)
    for at in _places(n):
        assert torch.equal(codes[at], Q.qadc_pq_encode(codebooks, x[at].contiguous())), at


@pytest.mark.parametrize("K", [5, 300])
def test_cells_of_many_vectors(K, memory_back):
    import paper_1704_07355_amd as Q
    n = (1 << 31) + 1234
    coarse = torch.randn((K, 2), generator=_gen(K), device=DEV)
    x = torch.empty((n, 2), device=DEV)
    for part in x.split(1 << 28):
        part.normal_(generator=_gen(3))
    cells = Q.qadc_ivf_assign(coarse, x)
    for at in _places(n):
        assert torch.equal(cells[at], Q.qadc_ivf_assign(coarse, x[at].contiguous())), at


def test_many_codes_between_the_layouts(memory_back):
    import paper_1704_07355_amd as Q
    n, half = MANY + 33, 16
    codes = torch.empty((n, half), dtype=torch.uint8, device=DEV)
    for part in codes.split(1 << 28):
        part.copy_(torch.randint(0, 256, (1 << 20, half), generator=_gen(4), dtype=torch.uint8, device=DEV).repeat(1 << 8, 1)[:len(part)])
    codes[-5000:] = torch.randint(0, 256, (5000, half), generator=_gen(5), dtype=torch.uint8, device=DEV)
    places = [slice(at.start // 16 * 16, at.stop) for at in _places(n, 960)]
    kept = [codes[at].clone() for at in places]
    packed = Q.qadc_pack_codes(codes, Q.QADC_LAYOUT_TRANSPOSED)
    for at, part in zip(places, kept):
        whole = len(part) // 16 * 16
        assert torch.equal(packed[at.start * half:(at.start + whole) * half], Q.qadc_pack_codes(part[:whole], Q.QADC_LAYOUT_TRANSPOSED)), at
    codes.zero_()
    Q.qadc_unpack_codes(packed, n, 2 * half, Q.QADC_LAYOUT_TRANSPOSED, out=codes)
    for at, part in zip(places, kept):
        assert torch.equal(codes[at], part), at


def test_centroids_of_many_cells(memory_back):
    import paper_1704_07355_amd as Q
    K, half = 8192, 33
    halves = torch.randn((2, K, half), generator=_gen(6), device=DEV)
    cells = Q.qadc_multi_index_cells(halves).view(K, K, 2 * half)
    for i in range(0, K, 256):
        part = cells[i:i + 256]
        same = torch.equal(part[:, :, :half], halves[0, i:i + 256, None].expand(256, K, half))
        same = same and torch.equal(part[:, :, half:], halves[1, None].expand(256, K, half))
        assert same, i


def test_lists_of_many_cells(memory_back):
    import paper_1704_07355_amd as Q
    n = MANY + 500
    cell_ids = torch.arange(0, 2000, 2, dtype=torch.int32, device=DEV)
    cells = torch.empty((n,), dtype=torch.int32, device=DEV)
    for part in cells.split(1 << 28):
        part.random_(-2, 2000, generator=_gen(7))
    slots = Q.qadc_multi_index_slots(cell_ids, cells)
    for a, b in zip(cells.split(1 << 28), slots.split(1 << 28)):
        same = torch.equal(b, torch.where((a >= 0) & (a % 2 == 0), a // 2, -1).to(torch.int32))
        assert same


def test_training_on_many_vectors(memory_back):
    """One step of Lloyd's algorithm from centroids 0 to 15, on sub-vectors that lie on them but for the last rows, beside the last one."""
    import paper_1704_07355_amd as Q
    n, m, ksub, more = 1 << 28, 16, 16, 4096
    x = torch.empty((n + more, m), device=DEV)
    for part in x[:n].split(1 << 24):
        part.random_(0, ksub, generator=_gen(8))
    x[n:] = ksub - 0.75
    x[torch.arange(ksub, device=DEV) + 7] = torch.arange(ksub, device=DEV)[:, None].float()
    count = torch.zeros((m,), dtype=torch.float64, device=DEV)
    for part in x[:n].split(1 << 24):
        count += (part == ksub - 1).sum(0)
    got = Q.qadc_pq_train(x, m, ksub, torch.arange(ksub, device=DEV) + 7, 1)[:, :, 0].double()
    want = torch.arange(ksub, dtype=torch.float64, device=DEV).repeat(m, 1)
    want[:, -1] = (count * (ksub - 1) + more * (ksub - 0.75)) / (count + more)
    assert ((got - want).abs() <= want * 2.0 ** -24 + 2.0 ** -40).all()
