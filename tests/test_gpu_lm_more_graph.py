"""A decode step and a training step of the norms, adapters, logit rules and distillation, as they are used together: captured in graphs
and replayed, on a stream of their own, and one after the other in a workspace that two graphs share."""

import pytest

import torch

from lm_common import DEV, gen

pytestmark = pytest.mark.gpu

ROWS, D, V, R, K_STORED = 6, 256, 3001, 8, 20


class Decode:
    """The state of a batch of requests, with a place for every input, so that a graph can be replayed on new ones."""

    def __init__(self):
        import paper_1704_07355_amd as Q
        g = gen(3)
        rand = lambda *s: torch.randn(s, generator=g, device=DEV)
        self.x = torch.empty((ROWS, D), dtype=torch.bfloat16, device=DEV)
        self.residual = torch.empty_like(self.x)
        self.weight = 1.0 + 0.1 * rand(D)
        codes = torch.randint(0, 256, (V, D // 2), generator=g, device=DEV, dtype=torch.uint8)
        self.head = Q.qadc_pack_weights4(codes, (0.01 + 0.01 * rand(V, D // 128).abs()).to(torch.bfloat16), None, D, 128)
        self.adapters = Q.qadc_adapters((rand(4, R, D) / 16).bfloat16(), rand(4, V, R).bfloat16(), rand(4).abs(),
                                        torch.tensor([8, 3, 8, 5], dtype=torch.int32, device=DEV))
        self.ids = torch.empty(ROWS, dtype=torch.int32, device=DEV)
        self.history = torch.empty((ROWS, 50), dtype=torch.int32, device=DEV)
        self.lengths = torch.empty(ROWS, dtype=torch.int32, device=DEV)
        self.penalty = torch.full((ROWS,), 1.2, device=DEV)
        self.frequency = torch.full((ROWS,), 0.3, device=DEV)
        self.bias_tokens = torch.randint(0, V, (ROWS, 5), generator=g, device=DEV, dtype=torch.int32)
        self.bias = rand(ROWS, 5)
        self.masks = torch.randint(-2 ** 31, 2 ** 31 - 1, (3, -(-V // 32)), generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
        self.mask_of = torch.empty(ROWS, dtype=torch.int32, device=DEV)
        self.ws = torch.empty(max(Q.qadc_adapters_workspace_bytes(self.adapters, ROWS), Q.qadc_token_logprobs_workspace_bytes(ROWS, V, 10)),
                              dtype=torch.uint8, device=DEV)

    def fill(self, seed):
        g = gen(seed)
        self.x.copy_(torch.randn((ROWS, D), generator=g, device=DEV))
        self.residual.copy_(torch.randn((ROWS, D), generator=g, device=DEV))
        self.ids.copy_(torch.randint(-1, 4, (ROWS,), generator=g, device=DEV))
        self.history.copy_(torch.randint(-1, V, self.history.shape, generator=g, device=DEV))
        self.lengths.copy_(torch.randint(0, 51, (ROWS,), generator=g, device=DEV))
        self.mask_of.copy_(torch.randint(-1, 3, (ROWS,), generator=g, device=DEV))

    def step(self):
        import paper_1704_07355_amd as Q
        state, total, _, rstd = Q.qadc_rms_norm(self.x, self.weight, self.residual)
        small, _, scale, _ = Q.qadc_rms_norm(self.x, self.weight, self.residual, out_type=torch.float8_e4m3fn)
        logits = Q.qadc_linear4(self.head, state)
        adapted = Q.qadc_add_adapters(self.adapters, self.ids, state, logits, workspace=self.ws)
        ruled = Q.qadc_adjust_logits(adapted, self.history, self.lengths, None, self.penalty, None, self.frequency, self.bias_tokens,
                                     self.bias, self.masks, self.mask_of)
        logp, lse, entropy, top, top_logp = Q.qadc_token_logprobs(ruled, k=10, workspace=self.ws)
        return state, total, rstd, small.view(torch.uint8), scale, adapted, ruled, lse, entropy, top, top_logp


class Train:
    """A student's norm and head, distilled from stored logits."""

    def __init__(self, rows):
        import paper_1704_07355_amd as Q
        g = gen(4)
        self.rows = rows
        self.x = torch.empty((rows, D), dtype=torch.bfloat16, device=DEV)
        self.residual = torch.empty_like(self.x)
        self.weight = 1.0 + 0.1 * torch.randn((D,), generator=g, device=DEV)
        self.head = (0.2 * torch.randn((V, D), generator=g, device=DEV)).bfloat16()
        self.back = self.head.t().contiguous()
        self.top = torch.empty((rows, K_STORED), dtype=torch.int32, device=DEV)
        self.top_logp = torch.empty((rows, K_STORED), device=DEV)
        self.share = torch.empty((rows,), device=DEV)
        self.ws = torch.empty(max(Q.qadc_distill_workspace_bytes(rows, V), Q.qadc_rms_norm_workspace_bytes(rows, D)), dtype=torch.uint8, device=DEV)

    def fill(self, seed):
        g = gen(seed)
        for t in (self.x, self.residual):
            t.copy_(torch.randn((self.rows, D), generator=g, device=DEV))
        lp = torch.log_softmax(2.0 * torch.randn((self.rows, V), generator=g, device=DEV), 1).topk(K_STORED, dim=1)
        self.top.copy_(lp.indices)
        self.top_logp.copy_(lp.values)
        self.share.copy_(torch.rand((self.rows,), generator=g, device=DEV))
        self.share[:2] = 0.0  # padding

    def step(self):
        import paper_1704_07355_amd as Q
        state, total, _, rstd = Q.qadc_rms_norm(self.x, self.weight, self.residual)
        logits = torch.mm(state, self.back)
        loss, lse, log_tail = Q.qadc_distill(logits, self.top, self.top_logp, workspace=self.ws)
        one = Q.qadc_distill_backward(logits, self.top, self.top_logp, lse, log_tail, self.share)
        both, dlogits = Q.qadc_distill_step(logits, self.top, self.top_logp, self.share, workspace=self.ws)
        dstate = torch.mm(dlogits, self.head)
        dx, dweight = Q.qadc_rms_norm_backward(dstate, total, self.weight, rstd, state, workspace=self.ws)
        return loss, lse, log_tail, one, both, dlogits, dx, dweight


def _same(a, b):
    return all(torch.equal(p.view(torch.uint8) if p.is_floating_point() else p, q.view(torch.uint8) if q.is_floating_point() else q)
               for p, q in zip((t.contiguous() for t in a), (t.contiguous() for t in b)))


@pytest.mark.parametrize("make", [Decode, lambda: Train(5), lambda: Train(200)], ids=["decode", "train5", "train200"])
def test_replays_equal_eager_calls(make):
    work = make()
    work.fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work.step()
    torch.cuda.current_stream().wait_stream(side)
    graphs, outputs = [], []
    for _ in range(2):  # two graphs that share the workspace, replayed one after the other
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outputs.append(work.step())
        graphs.append(graph)
    for seed in range(1, 6):
        work.fill(seed)
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        want = work.step()
        torch.cuda.synchronize()
        assert _same(outputs[0], want) and _same(outputs[1], want), seed


@pytest.mark.parametrize("make", [Decode, lambda: Train(200)], ids=["decode", "train200"])
def test_on_a_stream_of_its_own(make):
    work = make()
    work.fill(7)
    torch.cuda.synchronize()
    want = work.step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        busy = torch.randn((2048, 2048), device=DEV)
        for _ in range(5):
            busy = torch.mm(busy, busy) * 1e-3
        work.fill(8)
        work.fill(7)  # written on this stream, behind the products
        got = work.step()
    side.synchronize()
    assert _same(got, want)


def test_two_streams_with_a_workspace_each():
    a, b = Train(150), Train(150)
    a.fill(1)
    b.fill(2)
    want_a, want_b = a.step(), b.step()
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(one):
            got_a = a.step()
        with torch.cuda.stream(two):
            got_b = b.step()
        torch.cuda.synchronize()
        assert _same(got_a, want_a) and _same(got_b, want_b)


def test_a_padded_batch_gives_what_its_rows_give():
    """Rows behind the last sequence: every operator's row stands for itself."""
    import paper_1704_07355_amd as Q
    work = Decode()
    work.fill(5)
    full = work.step()
    n = 4
    state, total, _, rstd = Q.qadc_rms_norm(work.x[:n], work.weight, work.residual[:n])
    assert torch.equal(state, full[0][:n]) and torch.equal(total, full[1][:n])
    ruled = Q.qadc_adjust_logits(full[5][:n], work.history[:n], work.lengths[:n], None, work.penalty[:n], None, work.frequency[:n],
                                 work.bias_tokens[:n], work.bias[:n], work.masks, work.mask_of[:n])
    assert torch.equal(ruled, full[6][:n])
    room = torch.full((ROWS, V), 7.0, dtype=torch.bfloat16, device=DEV)
    Q.qadc_add_adapters(work.adapters, work.ids[:n], state, torch.zeros((n, V), dtype=torch.bfloat16, device=DEV), out=room[:n])
    assert (room[n:] == 7.0).all()


def test_the_rows_of_a_shorter_batch_have_the_bits_of_the_longer_one():
    """The first rows alone, beside rows that hold something else: outputs in 8 bits, adapters on the shared product, log probabilities."""
    import paper_1704_07355_amd as Q
    work = Decode()
    work.fill(6)
    state, total, rstd, small, scale, adapted, ruled, lse, entropy, top, top_logp = work.step()
    logits = Q.qadc_linear4(work.head, state)
    for n in (1, 4, 5):
        q, _, s, r = Q.qadc_rms_norm(work.x[:n], work.weight, work.residual[:n], out_type=torch.float8_e4m3fn)
        assert torch.equal(q.view(torch.uint8), small[:n]) and torch.equal(s, scale[:n]) and torch.equal(r, rstd[:n])
        room = torch.full((ROWS, V), 7.0, dtype=torch.bfloat16, device=DEV)
        Q.qadc_add_adapters(work.adapters, work.ids[:n], state[:n], logits[:n], out=room[:n], workspace=work.ws)
        # (256 inputs are not cut, for however many rows)
        assert torch.equal(room[:n], adapted[:n]) and (room[n:] == 7.0).all()
        got = Q.qadc_token_logprobs(ruled[:n], k=10, workspace=work.ws)
        assert _same(got[1:], (lse[:n], entropy[:n], top[:n], top_logp[:n]))
