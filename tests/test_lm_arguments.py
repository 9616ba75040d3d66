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
