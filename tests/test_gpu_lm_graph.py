"""The operators of a decode step captured in one graph and replayed: every replay equals the eager calls on the same inputs."""

import pytest

import torch

from lm_common import DEV, gen

pytestmark = pytest.mark.gpu


def test_a_decode_step_in_a_graph():
    import paper_1704_07355_amd as Q
    rows, d, V, R, T, k = 5, 640, 3001, 40, 7, 10
    g = gen(3)
    x = torch.empty((rows, d), dtype=torch.bfloat16, device=DEV)
    dist = torch.empty((rows, R), device=DEV)
    ids = torch.empty((rows, R), dtype=torch.int32, device=DEV)
    tokens = torch.randint(0, V, (rows, T), generator=g, device=DEV, dtype=torch.int32)
    weight, bias = torch.randn((2, d), generator=g, device=DEV).unbind(0)
    codes = torch.randint(0, 256, (V, d // 2), generator=g, device=DEV, dtype=torch.uint8)
    scales = (0.02 * torch.randn((V, d // 128), generator=g, device=DEV)).to(torch.bfloat16)
    head = Q.qadc_pack_weights4(codes, scales, None, d, 128)
    values = torch.randint(0, V, (1000,), generator=g, device=DEV, dtype=torch.int32)
    workspace = torch.empty(Q.qadc_token_logprobs_workspace_bytes(rows, V, k), dtype=torch.uint8, device=DEV)

    def fill(seed):
        h = gen(seed)
        x.copy_(torch.randn((rows, d), generator=h, device=DEV))
        dist.copy_(100.0 * torch.rand((rows, R), generator=h, device=DEV))
        ids.copy_(torch.randint(0, 1000, (rows, R), generator=h, device=DEV, dtype=torch.int32))

    def step():
        y = Q.qadc_layer_norm(x, weight, bias)[0]
        logits = Q.qadc_linear4(head, y)
        logp, lse, entropy, top, top_logp = Q.qadc_token_logprobs(logits, tokens, k, 0.8, workspace=workspace)
        mix, knn = Q.qadc_neighbour_mix(ids, dist, values, tokens, logp, 0.3, 0.05)
        return logits, logp, lse, entropy, top, top_logp, mix, knn

    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in range(1, 5):
        fill(seed)
        graph.replay()
        torch.cuda.synchronize()
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), seed
