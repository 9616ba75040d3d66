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
    assert size(17, 129, 32, 1) == 4 * 1024 + 2 * 5 * 48
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
