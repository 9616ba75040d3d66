"""The norms, logit rules, distillation and adapters check their arguments on the host, before anything is launched (no GPU needed)."""

import paper_1704_07355_amd as Q

PTR = 256  # stands for a device pointer: every call below is refused before it is used


def test_rms_norm():
    L = Q.lib()
    ok = dict(x=PTR, ldx=8, res=None, ldr=0, type=0, w=None, wtype=0, rows=3, d=8, eps=1e-5, sum=None, ld_sum=0, y=2 * PTR, ytype=0,
              scale=None, rstd=None, stream=None)

    def f(**k):
        return L.qadc_rms_norm(*dict(ok, **k).values())

    assert f(x=None, y=None, rows=0) == Q.QADC_OK  # nothing to do
    for bad in (dict(x=None), dict(y=None), dict(type=3), dict(type=-1), dict(wtype=2), dict(rows=-1), dict(d=0), dict(d=2 ** 31 - 1),
                dict(ldx=7), dict(eps=float("nan")), dict(eps=-1.0), dict(ytype=1), dict(ytype=3), dict(ytype=3, y=PTR, scale=PTR),
                dict(res=3 * PTR, ldr=8), dict(res=3 * PTR, ldr=7, sum=4 * PTR, ld_sum=8), dict(res=3 * PTR, ldr=8, sum=4 * PTR, ld_sum=7),
                dict(res=3 * PTR, ldr=9, sum=3 * PTR, ld_sum=8), dict(res=3 * PTR, ldr=8, sum=PTR, ld_sum=9),
                dict(res=3 * PTR, ldr=8, sum=2 * PTR, ld_sum=8), dict(y=PTR, ldx=9), dict(res=2 * PTR, ldr=9, sum=4 * PTR, ld_sum=8)):
        assert f(**bad) == Q.QADC_EINVAL, bad
    assert b"qadc_rms_norm" in L.qadc_last_error()


def test_rms_norm_backward():
    L = Q.lib()
    need = Q.qadc_rms_norm_workspace_bytes(100, 8)
    assert need > 0 and Q.qadc_rms_norm_workspace_bytes(-1, 8) == 0 and Q.qadc_rms_norm_workspace_bytes(4, 0) == 0
    ok = dict(dy=PTR, lddy=8, ds=None, ldds=0, h=2 * PTR, ldh=8, type=0, w=None, wtype=0, rstd=PTR, rows=100, d=8, dx=3 * PTR, dw=PTR,
              ws=PTR, size=need, stream=None)

    def f(**k):
        return L.qadc_rms_norm_backward(*dict(ok, **k).values())

    assert f(size=0) == Q.QADC_ENOMEM and f(ws=None) == Q.QADC_ENOMEM
    for bad in (dict(dy=None), dict(h=None), dict(rstd=None), dict(lddy=7), dict(ldh=7), dict(ds=PTR, ldds=7), dict(type=3),
                dict(wtype=1), dict(rows=-1), dict(d=0), dict(dx=PTR, lddy=9), dict(dx=2 * PTR, ldh=9),
                dict(ds=3 * PTR, ldds=9), dict(ws=PTR + 8)):
        assert f(**bad) == Q.QADC_EINVAL, bad
    assert b"qadc_rms_norm_backward" in L.qadc_last_error()


def test_adjust_logits():
    L = Q.lib()
    ok = dict(x=PTR, ld=64, type=0, rows=3, V=64, history=None, H=0, lengths=None, prompt=None, rep=None, pres=None, freq=None,
              bt=None, bias=None, B=0, masks=None, ldm=0, states=0, of=None, out=2 * PTR, ldo=64, stream=None)

    def f(**k):
        return L.qadc_adjust_logits(*dict(ok, **k).values())

    assert f(x=None, out=None, rows=0) == Q.QADC_OK
    for bad in (dict(x=None), dict(out=None), dict(type=3), dict(rows=-1), dict(V=0), dict(V=2 ** 31 - 1, ld=2 ** 31, ldo=2 ** 31),
                dict(ld=63), dict(ldo=63), dict(H=5), dict(H=-1), dict(H=Q.QADC_MAX_HISTORY + 1, history=PTR), dict(B=2, bt=PTR),
                dict(B=2, bias=PTR), dict(B=Q.QADC_MAX_R + 1, bt=PTR, bias=PTR), dict(B=-1), dict(masks=PTR, ldm=1, states=3),
                dict(masks=PTR, ldm=2, states=0), dict(masks=PTR, ldm=2, states=2), dict(out=PTR, ldo=65)):
        assert f(**bad) == Q.QADC_EINVAL, bad
    assert b"qadc_adjust_logits" in L.qadc_last_error()


def test_distill():
    L = Q.lib()
    need = Q.qadc_distill_workspace_bytes(3, 100000)
    assert need > 0 and Q.qadc_distill_workspace_bytes(0, 10) == 0 and Q.qadc_distill_workspace_bytes(3, 0) == 0
    ok = dict(x=PTR, ld=100000, type=0, rows=3, V=100000, scale=1.0, idx=PTR, logp=PTR, k=5, tail=1)
    loss = dict(loss=PTR, lse=PTR, log_tail=PTR, ws=PTR, size=need, stream=None)
    grad = dict(lse=PTR, log_tail=PTR, dloss=PTR, out=2 * PTR, ldo=100000, stream=None)
    step = dict(weight=PTR, loss=PTR, out=2 * PTR, ldo=100000, ws=PTR, size=need, stream=None)
    for name, more, own in (("qadc_distill", loss, (dict(loss=None),)),
                            ("qadc_distill_backward", grad, (dict(lse=None), dict(log_tail=None), dict(dloss=None), dict(out=None),
                                                             dict(ldo=99999), dict(out=PTR, ldo=100001))),
                            ("qadc_distill_step", step, (dict(weight=None), dict(loss=None), dict(out=None), dict(ldo=99999),
                                                         dict(out=PTR, ldo=100001)))):
        def f(**k):
            return getattr(L, name)(*{**ok, **more, **k}.values())

        assert f(x=None, rows=0) == Q.QADC_OK
        for bad in (dict(x=None), dict(type=3), dict(rows=-1), dict(V=0), dict(V=2 ** 31 - 1, ld=2 ** 31), dict(ld=99999), dict(scale=0.0),
                    dict(scale=float("nan")), dict(scale=3e38), dict(k=-1), dict(k=129), dict(idx=None), dict(logp=None)) + own:
            assert f(**bad) == Q.QADC_EINVAL, (name, bad)
        assert name.encode() + b":" in L.qadc_last_error()
        if "ws" in more:
            assert f(ws=None) == Q.QADC_ENOMEM and f(size=16) == Q.QADC_ENOMEM and f(ws=PTR + 8) == Q.QADC_EINVAL


def test_add_adapters():
    import ctypes
    L = Q.lib()

    def pool(**k):
        w = Q.qadc_adapters.__new__(Q.qadc_adapters)
        for name, v in dict(dict(a=PTR, b=PTR, N=500, K=3000, rank=16, count=4, type=1), **k).items():
            setattr(w, name, v)
        return w

    w = pool()
    need = Q.qadc_adapters_workspace_bytes(w, 64)
    assert need > 0 and Q.qadc_adapters_workspace_bytes(w, 0) == 0
    assert all(Q.qadc_adapters_workspace_bytes(w, m) <= Q.qadc_adapters_workspace_bytes(w, 5000) for m in range(1, 5000, 37))
    ok = dict(w=w, ids=PTR, x=PTR, ldx=3000, M=64, base=2 * PTR, ldb=500, y=3 * PTR, ldy=500, ws=PTR, size=need, stream=None)

    def f(**k):
        a = dict(ok, **k)
        a["w"] = None if a["w"] is None else ctypes.byref(a["w"])
        return L.qadc_add_adapters(*a.values())

    assert f(M=0, ids=None, x=None, y=None) == Q.QADC_OK
    for bad in (dict(w=None), dict(ids=None), dict(x=None), dict(y=None), dict(ldx=2999), dict(ldb=499), dict(ldy=499), dict(M=-1),
                dict(M=(1 << 24) + 1), dict(y=2 * PTR, ldb=501), dict(ws=PTR + 8)):
        assert f(**bad) == Q.QADC_EINVAL, bad
    for k, v in (("a", None), ("b", None), ("N", 0), ("N", (1 << 30) + 1), ("K", 0), ("rank", 0), ("rank", 129), ("count", 0), ("type", 3)):
        assert f(w=pool(**{k: v}), ldx=1 << 25, ldb=1 << 31, ldy=1 << 31) == Q.QADC_EINVAL, (k, v)
    assert f(ws=None) == Q.QADC_ENOMEM and f(size=16) == Q.QADC_ENOMEM
    assert b"qadc_add_adapters" in L.qadc_last_error()
    # more workgroups than a launch takes
    assert f(w=pool(N=1 << 30, count=300), M=1 << 24, ldb=1 << 30, ldy=1 << 30, size=1 << 40) == Q.QADC_EINVAL


def test_add_adapters_takes_as_many_rows_and_outputs_as_it_says():
    """ceil(M / 256) * ceil(N / 2048) < 2^24 on both sides, with adapters that leave rows single and with few; a call that is not refused for its
    size goes on to its workspace, which is too small."""
    import ctypes
    L = Q.lib()

    def f(M, N, count):
        w = Q.qadc_adapters.__new__(Q.qadc_adapters)
        for name, v in dict(a=PTR, b=PTR, N=N, K=64, rank=16, count=count, type=1).items():
            setattr(w, name, v)
        return L.qadc_add_adapters(ctypes.byref(w), PTR, PTR, 64, M, None, 0, 3 * PTR, N, PTR, 16, None)

    for count in (1, 4, 300, 2000, 1 << 20):
        for M, N in ((4096, 1 << 24), (65536, 1 << 20), (256, 1 << 27), (256, (1 << 27) + 2048), (255, 1 << 30), (1 << 24, 1), (1 << 24, 255 * 2048),
                     (31 * 256, 1 << 30), ((1 << 24) - 300, 255 * 2048 - 1), (4097 * 256, 4094 * 2048), (1, 1 << 30), (3000 * 256, 5000 * 2048)):
            assert f(M, N, count) == Q.QADC_ENOMEM, (M, N, count)
        for M, N in ((1 << 24, 256 * 2048), (32 * 256, 1 << 30), (4096 * 256, 4096 * 2048), (31 * 256 + 1, 1 << 30), (1 << 24, 255 * 2048 + 1),
                     (1 << 24, 1 << 30)):
            assert f(M, N, count) == Q.QADC_EINVAL, (M, N, count)
