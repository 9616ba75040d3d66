"""The language-model operators check their arguments on the host, before anything is launched (no GPU needed)."""

import paper_1704_07355_amd as Q

PTR = 256  # stands for a device pointer: every call below is refused before it is used


def test_layer_norm():
    L = Q.lib()
    f = L.qadc_layer_norm
    assert f(None, 8, 0, None, None, 0, 0, 8, 1e-5, None, None, None, None) == Q.QADC_OK        # nothing to do
    assert f(None, 8, 0, None, None, 0, 3, 8, 1e-5, PTR, None, None, None) == Q.QADC_EINVAL     # null pointer
    assert f(PTR, 8, 3, None, None, 0, 3, 8, 1e-5, PTR, None, None, None) == Q.QADC_EINVAL      # unknown type
    assert f(PTR, 8, 1, None, None, 2, 3, 8, 1e-5, PTR, None, None, None) == Q.QADC_EINVAL      # weight of a third type
    assert f(PTR, 7, 0, None, None, 0, 3, 8, 1e-5, PTR, None, None, None) == Q.QADC_EINVAL      # rows overlap
    assert f(PTR, 8, 0, None, None, 0, -1, 8, 1e-5, PTR, None, None, None) == Q.QADC_EINVAL
    assert f(PTR, 8, 0, None, None, 0, 3, 0, 1e-5, PTR, None, None, None) == Q.QADC_EINVAL
    assert f(PTR, 8, 0, None, None, 0, 3, 8, float("nan"), PTR, None, None, None) == Q.QADC_EINVAL
    assert f(PTR, 9, 0, None, None, 0, 3, 8, 1e-5, PTR, None, None, None) == Q.QADC_EINVAL      # in place with rows apart
    assert b"qadc_layer_norm" in L.qadc_last_error()


def test_layer_norm_backward():
    L = Q.lib()
    need = Q.qadc_layer_norm_workspace_bytes(100, 8)
    assert need > 0 and Q.qadc_layer_norm_workspace_bytes(-1, 8) == 0 and Q.qadc_layer_norm_workspace_bytes(4, 0) == 0
    f = L.qadc_layer_norm_backward
    assert f(PTR, 8, PTR, 8, 0, None, 0, PTR, PTR, 100, 8, PTR, PTR, PTR, PTR, need - 1, None) == Q.QADC_ENOMEM
    assert f(PTR, 8, PTR, 8, 0, None, 0, PTR, PTR, 100, 8, PTR, PTR, PTR, None, need, None) == Q.QADC_ENOMEM
    assert f(PTR, 8, PTR, 8, 0, None, 0, None, PTR, 100, 8, PTR, PTR, PTR, PTR, need, None) == Q.QADC_EINVAL
    assert f(PTR, 8, PTR, 7, 0, None, 0, PTR, PTR, 100, 8, PTR, PTR, PTR, PTR, need, None) == Q.QADC_EINVAL
    assert f(PTR, 9, PTR + 8, 8, 0, None, 0, PTR, PTR, 100, 8, PTR, PTR, PTR, PTR, need, None) == Q.QADC_EINVAL  # dx = dy, apart
    assert f(PTR, 8, PTR, 8, 7, None, 0, PTR, PTR, 100, 8, PTR, PTR, PTR, PTR, need, None) == Q.QADC_EINVAL


def test_weights4_and_linear4():
    import ctypes
    L = Q.lib()
    size = Q.qadc_weights4_bytes
    assert size(16, 128, 128, 0) == 1024 + 32 and size(16, 128, 128, 1) == 1024 + 48
    assert size(17, 129, 32, 1) == 4 * 1024 + 2 * 2 * 4 * 48  # the groups of a tile's inputs lie together
    assert size(17, 129, 256, 1) == 4 * 1024 + 2 * 48
    for bad in ((0, 128, 128, 0), (16, 0, 128, 0), (16, (1 << 24) + 1, 128, 0), (16, 128, 48, 0), (16, 128, 0, 0), (16, 128, 192, 0),
                (1 << 31, 128, 128, 0)):
        assert size(*bad) == 0
    f = L.qadc_pack_weights4
    assert f(PTR, PTR, 0, None, 16, 128, 128, PTR, None) == Q.QADC_EINVAL      # float32 scales
    assert f(None, PTR, 1, None, 16, 128, 128, PTR, None) == Q.QADC_EINVAL
    assert f(PTR, PTR, 1, None, 16, 128, 128, PTR + 8, None) == Q.QADC_EINVAL  # not aligned
    w = Q.qadc_weights4(PTR, 16, 128, 128, 1, 0)
    g = lambda w, *a: L.qadc_linear4(None if w is None else ctypes.byref(w), *a)
    assert g(w, None, 128, 0, 0, None, None, 16, None) == Q.QADC_OK            # nothing to do
    assert g(None, PTR, 128, 0, 1, None, PTR, 16, None) == Q.QADC_EINVAL
    assert g(w, None, 128, 0, 1, None, PTR, 16, None) == Q.QADC_EINVAL
    assert g(w, PTR, 127, 0, 1, None, PTR, 16, None) == Q.QADC_EINVAL
    assert g(w, PTR, 128, 0, 1, None, PTR, 15, None) == Q.QADC_EINVAL
    assert g(w, PTR, 128, 5, 1, None, PTR, 16, None) == Q.QADC_EINVAL
    assert g(w, PTR, 128, 0, -1, None, PTR, 16, None) == Q.QADC_EINVAL
    for field, value in (("packed", None), ("group", 100), ("stype", 0), ("N", 0), ("K", 0)):
        bad = Q.qadc_weights4(PTR, 16, 128, 128, 1, 0)
        setattr(bad, field, value)
        assert g(bad, PTR, 128, 0, 1, None, PTR, 16, None) == Q.QADC_EINVAL
    assert b"qadc_linear4" in L.qadc_last_error()


def test_weights4_of_too_many_outputs():
    """Beyond 2^30 outputs the threads of a product's grid would pass 32 bits."""
    assert Q.qadc_weights4_bytes(1 << 30, 128, 128, 0) == (1 << 26) * (1024 + 32)
    assert Q.qadc_weights4_bytes((1 << 30) + 1, 128, 128, 0) == 0


def test_token_logprobs():
    L = Q.lib()
    need = Q.qadc_token_logprobs_workspace_bytes(4, 1000, 10)
    assert need > 0
    for bad in ((0, 1000, 10), (4, 0, 10), (4, 1000, -1), (4, 1000, 129)):
        assert Q.qadc_token_logprobs_workspace_bytes(*bad) == 0
    P = PTR
    f = L.qadc_token_logprobs
    assert f(None, 1000, 0, 0, 1000, 1.0, None, 0, 0, None, None, None, None, None, None, 0, None) == Q.QADC_OK
    ok = [P, 1000, 0, 4, 1000, 1.0, P, 2, 10, P, P, P, P, P, P, need, None]
    for at, value, code in ((0, None, Q.QADC_EINVAL), (1, 999, Q.QADC_EINVAL), (2, 3, Q.QADC_EINVAL), (3, -1, Q.QADC_EINVAL),
                            (4, 0, Q.QADC_EINVAL), (5, 0.0, Q.QADC_EINVAL), (5, float("nan"), Q.QADC_EINVAL), (6, None, Q.QADC_EINVAL),
                            (7, -1, Q.QADC_EINVAL), (7, 1025, Q.QADC_EINVAL), (8, 129, Q.QADC_EINVAL), (9, None, Q.QADC_EINVAL),
                            (12, None, Q.QADC_EINVAL), (13, None, Q.QADC_EINVAL), (14, None, Q.QADC_ENOMEM), (15, need - 1, Q.QADC_ENOMEM)):
        args = list(ok)
        args[at] = value
        assert f(*args) == code, (at, value)
    assert b"qadc_token_logprobs" in L.qadc_last_error()
    g = L.qadc_token_logprobs_backward
    assert g(None, 1000, 0, 0, 1000, 1.0, None, 0, None, None, None, None, None, 1000, None) == Q.QADC_OK
    ok = [P, 1000, 0, 4, 1000, 1.0, P, 2, P, P, P, P, P + 256, 1000, None]
    for at, value in ((0, None), (1, 999), (2, -1), (5, -1.0), (6, None), (7, 1025), (8, None), (9, None), (10, None), (12, None), (13, 999)):
        args = list(ok)
        args[at] = value
        assert g(*args) == Q.QADC_EINVAL, (at, value)
    assert g(P, 1000, 0, 4, 1000, 1.0, P, 2, P, P, P, P, P, 1001, None) == Q.QADC_EINVAL  # in place, other row distances


def test_token_logprobs_scale_beyond_the_exponent():
    """A scale whose product with log2(e) is no float32 would turn 0 times it into NaN."""
    L = Q.lib()
    P = PTR
    need = Q.qadc_token_logprobs_workspace_bytes(4, 1000, 10)
    assert L.qadc_token_logprobs(P, 1000, 0, 4, 1000, 3e38, P, 2, 10, P, P, P, P, P, P, need, None) == Q.QADC_EINVAL
    assert L.qadc_token_logprobs_backward(P, 1000, 0, 4, 1000, 3e38, P, 2, P, P, P, P, P + 256, 1000, None) == Q.QADC_EINVAL
    assert L.qadc_token_logprobs(None, 1000, 0, 0, 1000, 2e38, None, 0, 0, None, None, None, None, None, None, 0, None) == Q.QADC_OK


def test_neighbour_mix():
    L = Q.lib()
    P = PTR
    f = L.qadc_neighbour_mix
    assert f(None, None, 4, None, 0, 10, None, 5, 1.0, None, 3, None, 0.5, None, None, None) == Q.QADC_OK
    assert f(None, None, 4, None, 2, 10, None, 5, 1.0, None, 0, None, 0.5, None, None, None) == Q.QADC_OK
    ok = [P, P, 4, None, 2, 10, P, 5, 1.0, P, 3, P, 0.5, P, P, None]
    for at, value in ((0, None), (1, None), (2, 2), (4, -1), (5, 0), (5, 1025), (6, None), (7, -1), (8, -0.5), (8, float("nan")), (9, None),
                      (10, -1), (11, None), (12, 1.1), (12, float("nan")), (13, None)):
        args = list(ok)
        args[at] = value
        assert f(*args) == Q.QADC_EINVAL, (at, value)
    assert b"qadc_neighbour_mix" in L.qadc_last_error()


def test_neighbour_mix_of_more_tokens_than_an_int_counts():
    """A row's tokens are counted in steps of up to 256: the last step must not pass 2^31."""
    f = Q.lib().qadc_neighbour_mix
    for T in (2 ** 31 - 1, 2 ** 31 - 1023):
        assert f(PTR, PTR, 4, None, 0, 10, PTR, 5, 1.0, PTR, T, PTR, 0.5, PTR, PTR, None) == Q.QADC_EINVAL
    assert f(PTR, PTR, 4, None, 0, 10, PTR, 5, 1.0, PTR, 2 ** 31 - 1025, PTR, 0.5, PTR, PTR, None) == Q.QADC_OK  # (no rows)


def test_layer_norm_of_longer_rows_than_an_int_counts():
    """A row's columns are counted in steps of a workgroup: the last step must not pass 2^31."""
    L = Q.lib()
    for d in (2 ** 31 - 1, 2 ** 31 - 1023):
        assert L.qadc_layer_norm(PTR, d, 1, None, None, 1, 0, d, 1e-5, PTR, None, None, None) == Q.QADC_EINVAL
        assert L.qadc_layer_norm_backward(PTR, d, PTR, d, 1, None, 1, PTR, PTR, 0, d, PTR, None, None, None, 0, None) == Q.QADC_EINVAL
    assert Q.qadc_layer_norm_workspace_bytes(4, 2 ** 31 - 1) == 0
    d = 2 ** 31 - 1025
    assert L.qadc_layer_norm(PTR, d, 1, None, None, 1, 0, d, 1e-5, PTR, None, None, None) == Q.QADC_OK  # (no rows)


def test_layer_norm_workspaces_grow_with_the_batch():
    """What is asked for a batch holds what is asked for any smaller one."""
    for d in (1, 100, 300, 900, 2000, 4096, 4097, 16384, 16385, 100000):
        sizes = [Q.qadc_layer_norm_workspace_bytes(rows, d) for rows in [*range(0, 2100), *range(2100, 40000, 37), 1 << 20, 1 << 33]]
        assert sizes == sorted(sizes) and sizes[1] > 0, d


def test_token_logprobs_workspaces_grow_with_the_call():
    """What is asked for a call holds what is asked for one of fewer rows, tokens or alternatives."""
    size = Q.qadc_token_logprobs_workspace_bytes
    rows_of, V_of = [*range(1, 600), 1000, 1023, 1024, 1025, 5000], [*range(1, 600000, 4095), 10 ** 6, 8400000, 8400000 + 8192, 10 ** 7]
    for k in (0, 1, 128):
        for V in (1, 5000, 8185, 8186, 20000, 60000, 131072, 262144, 390000, 400000, 10 ** 7):
            sizes = [size(rows, V, k) for rows in rows_of]
            assert sizes == sorted(sizes), (V, k)
            assert size(30, V, 0) <= size(30, V, 1) == size(30, V, 128)
        for rows in (1, 2, 3, 100, 399, 400, 2000):
            sizes = [size(rows, V, k) for V in V_of]
            assert sizes == sorted(sizes), (rows, k)
