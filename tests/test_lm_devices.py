"""Every tensor of a call of the norms in 8 bits, logit rules, distillation and adapters has to be on one GPU, the current one (no GPU needed:
the tensors only say that they are on one, and the library is not reached)."""

import pytest

import torch

import paper_1704_07355_amd as Q
from paper_1704_07355_amd import binding


class Placed(torch.Tensor):
    """A host tensor that says it is on GPU number `at`."""
    at = 0
    is_cuda = property(lambda self: True)

    def get_device(self):
        return self.at


def placed(t, at=0):
    with torch._C.DisableTorchFunctionSubclass():
        t = t.as_subclass(Placed)
    t.at = at
    return t


@pytest.fixture
def calls(monkeypatch):
    """The library's entry points, noted instead of called, and GPU 0 as the current one."""
    noted = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: noted.append(name) or 0

    empty, empty_like = torch.empty, torch.empty_like
    monkeypatch.setattr(binding, "lib", Library)
    monkeypatch.setattr(binding, "_raw_stream", lambda device: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: placed(empty(*a, **k)))
    monkeypatch.setattr(torch, "empty_like", lambda *a, **k: placed(empty_like(*a, **k)))
    return noted


ROWS, D, V, K, B, H = 3, 8, 40, 5, 2, 6
F32, I32, U8 = torch.float32, torch.int32, torch.uint8


def _z(*size, dtype=F32):
    return torch.zeros(size, dtype=dtype)


def _rms(t):
    return Q.qadc_rms_norm(t["x"], t["weight"], t["residual"], sum_out=t["sum_out"], out=t["out"])


def _rms8(t):
    return Q.qadc_rms_norm(t["x"], out_type=torch.float8_e4m3fn, out=t["out8"])


def _rms_backward(t):
    return Q.qadc_rms_norm_backward(t["dy"], t["h"], t["weight"], t["rstd"], t["dsum"], workspace=t["workspace"], out=t["out"])


def _adjust(t):
    return Q.qadc_adjust_logits(**t)


def _distill(t):
    return Q.qadc_distill(t["logits"], t["top_idx"], t["top_logp"], workspace=t["workspace"])


def _distill_backward(t):
    return Q.qadc_distill_backward(**t)


def _distill_step(t):
    return Q.qadc_distill_step(**t)


def _adapters(t):
    pool = Q.qadc_adapters(t["a"], t["b"], t["scales"], t["ranks"])
    return Q.qadc_add_adapters(pool, t["ids"], t["x"], t["base"], out=t["out"], workspace=t["workspace"])


TEACHER = dict(logits=_z(ROWS, V), top_idx=_z(ROWS, K, dtype=I32), top_logp=_z(ROWS, K))
CALLS = {
    "qadc_rms_norm": (_rms, dict(x=_z(ROWS, D), weight=_z(D), residual=_z(ROWS, D), sum_out=_z(ROWS, D), out=_z(ROWS, D))),
    "qadc_rms_norm to 8 bits": (_rms8, dict(x=_z(ROWS, D), out8=_z(ROWS, D).to(torch.float8_e4m3fn))),
    "qadc_rms_norm_backward": (_rms_backward, dict(dy=_z(ROWS, D), h=_z(ROWS, D), weight=_z(D), rstd=_z(ROWS), dsum=_z(ROWS, D),
                                                   workspace=_z(256, dtype=U8), out=_z(ROWS, D))),
    "qadc_adjust_logits": (_adjust, dict(logits=_z(ROWS, V), history=_z(ROWS, H, dtype=I32), lengths=_z(ROWS, dtype=I32),
                                         prompt=_z(ROWS, dtype=I32), repetition=_z(ROWS), presence=_z(ROWS), frequency=_z(ROWS),
                                         bias_tokens=_z(ROWS, B, dtype=I32), bias=_z(ROWS, B), masks=_z(4, 2, dtype=I32),
                                         mask_of=_z(ROWS, dtype=I32), out=_z(ROWS, V))),
    "qadc_distill": (_distill, dict(TEACHER, workspace=_z(256, dtype=U8))),
    "qadc_distill_backward": (_distill_backward, dict(TEACHER, lse=_z(ROWS), log_tail=_z(ROWS), dloss=_z(ROWS), out=_z(ROWS, V))),
    "qadc_distill_step": (_distill_step, dict(TEACHER, weight=_z(ROWS), out=_z(ROWS, V), workspace=_z(256, dtype=U8))),
    "qadc_add_adapters": (_adapters, dict(a=_z(2, 4, D), b=_z(2, V, 4), scales=_z(2), ranks=_z(2, dtype=I32), ids=_z(ROWS, dtype=I32),
                                          x=_z(ROWS, D), base=_z(ROWS, V), out=_z(ROWS, V), workspace=_z(256, dtype=U8))),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_a_tensor_on_another_gpu_is_refused(name, calls):
    call, tensors = CALLS[name]
    entry = name.split()[0]
    call({k: placed(t) for k, t in tensors.items()})
    assert calls.count(entry) == 1
    for stray in tensors:
        with pytest.raises(ValueError, match="cuda:1"):
            call({k: placed(t, int(k == stray)) for k, t in tensors.items()})
        with pytest.raises(ValueError):
            call({k: t if k == stray else placed(t) for k, t in tensors.items()})
    with pytest.raises(ValueError, match="cuda:1"):  # together, but not where the call would run
        call({k: placed(t, 1) for k, t in tensors.items()})
    assert calls.count(entry) == 1
