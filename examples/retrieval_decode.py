"""A language model's step over a datastore of its hidden states, and a training step of what comes before the search.

The datastore holds (state, token that followed) pairs: the states as 4-bit product-quantization codes, the tokens as a
table by id.  A decode step

  normalises the hidden states (qadc_layer_norm),
  multiplies them with the vocabulary head's 4-bit weights (qadc_linear4),
  searches the datastore for the nearest states (qadc_build_luts, qadc_quantize_luts, qadc_scan_topk),
  takes the log probabilities of the neighbours' tokens and the model's own likeliest ones (qadc_token_logprobs),
  and mixes the neighbours' votes in (qadc_neighbour_mix).

The training step fits the norm's weight and bias to the tokens that followed: the loss is the mean of -log p - gamma *
entropy, its gradient comes from qadc_token_logprobs_backward and qadc_layer_norm_backward (the head stays as it is).

All data is synthetic: every token has a prototype state, the model's head is a blurred copy of the prototypes, and
observed states scatter around theirs, each column with a scale and an offset of its own that the norm has to undo.

    python examples/retrieval_decode.py [--states 200000] [--batch 32] [--steps 40]
"""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1704_07355_amd as Q  # noqa: E402

DEV = "cuda:0"
D, M, VOCABULARY, GROUP = 128, 32, 8192, 32
R, ALTERNATIVES, INIT = 64, 16, 1000
LAMBDA, TEMPERATURE = 0.5, 10.0   # share of the neighbours, and the distance over which a vote falls to 1/e


def make_model(g):
    """Prototypes of the tokens [V][D], the head [V][D] that the model has of them, and the columns' scale and offset."""
    prototypes = torch.randn((VOCABULARY, D), generator=g, device=DEV)
    head = (prototypes + 2.0 * torch.randn((VOCABULARY, D), generator=g, device=DEV)) * 0.25
    scale = torch.exp(0.5 * torch.randn((D,), generator=g, device=DEV))
    offset = torch.randn((D,), generator=g, device=DEV)
    return prototypes, head, scale, offset


def observe(prototypes, scale, offset, n, g):
    """n hidden states (bfloat16) and the tokens that followed, drawn unevenly."""
    u = torch.rand((n,), generator=g, device=DEV)
    tokens = (u * u * VOCABULARY).to(torch.int32).clamp_(max=VOCABULARY - 1)
    x = prototypes[tokens.long()] + 0.6 * torch.randn((n, D), generator=g, device=DEV)
    return (x * scale + offset).bfloat16(), tokens


def quantize_head(head):
    """4-bit codes around a group's middle, binary16 scales and zero points, laid out for qadc_linear4."""
    w = head.reshape(VOCABULARY, D // GROUP, GROUP)
    lo, hi = w.amin(2), w.amax(2)
    scales = ((hi - lo) / 15).half()
    zeros = torch.round(-lo / scales.float()).clamp_(0, 15).to(torch.uint8)
    q = torch.round(w / scales.float()[..., None] + zeros[..., None]).clamp_(0, 15).to(torch.uint8).reshape(VOCABULARY, D)
    return Q.qadc_pack_weights4((q[:, 0::2] | q[:, 1::2] << 4).contiguous(), scales, zeros, D, GROUP)


def build_datastore(states):
    """Codebooks trained on the first states and the codes of all, from normalised states in float32."""
    train = states[:20000]
    init = torch.arange(16, device=DEV, dtype=torch.int64) * (train.shape[0] // 16)
    codebooks = Q.qadc_pq_train(train, M, 16, init, 8)
    return codebooks, Q.qadc_pq_encode(codebooks, states)


def decode(hidden, weight, bias, head, codebooks, codes, values):
    """One step of a batch -> (candidates i32 [B][C], their mixed log probabilities, the model's own)."""
    state, _, _ = Q.qadc_layer_norm(hidden, weight, bias)
    logits = Q.qadc_linear4(head, state)
    luts = Q.qadc_build_luts(codebooks, state.float())
    qluts, _, delta, _ = Q.qadc_quantize_luts(luts, codes[:INIT], R)
    ids, sums = Q.qadc_scan_topk(Q.QADC_U8_4BIT, codes, qluts, R)
    # the neighbours' tokens (an unused slot where there is no neighbour), then the model's own likeliest
    near = torch.where(ids >= 0, values[ids.clamp(min=0).long()], -1)
    logp, _, _, top, top_logp = Q.qadc_token_logprobs(logits, near, ALTERNATIVES)
    candidates = torch.cat((top, near), 1)
    own = torch.cat((top_logp, logp), 1)
    mixed, _ = Q.qadc_neighbour_mix(ids, sums, values, candidates, own, LAMBDA, 1 / TEMPERATURE, delta)
    return candidates, torch.where(candidates >= 0, mixed, -float("inf")), own


def score(hidden, targets, weight, bias, head, codebooks, codes, values):
    """Mean -log p of the tokens that followed: the model's own, and with the neighbours mixed in."""
    state, _, _ = Q.qadc_layer_norm(hidden, weight, bias)
    logits = Q.qadc_linear4(head, state)
    luts = Q.qadc_build_luts(codebooks, state.float())
    qluts, _, delta, _ = Q.qadc_quantize_luts(luts, codes[:INIT], R)
    ids, sums = Q.qadc_scan_topk(Q.QADC_U8_4BIT, codes, qluts, R)
    logp, _, _, _, _ = Q.qadc_token_logprobs(logits, targets[:, None].contiguous())
    mixed, _ = Q.qadc_neighbour_mix(ids, sums, values, targets[:, None].contiguous(), logp, LAMBDA, 1 / TEMPERATURE, delta)
    return -logp.mean().item(), -mixed.mean().item()


def train_step(hidden, targets, weight, bias, head, rate, gamma=0.01):
    """One step of gradient descent on the norm's weight and bias; returns the loss before it."""
    rows = hidden.shape[0]
    state, mean, rstd = Q.qadc_layer_norm(hidden, weight, bias)
    logits = (state.float() @ head.t()).bfloat16()
    tokens = targets[:, None].contiguous()
    logp, lse, entropy, _, _ = Q.qadc_token_logprobs(logits, tokens)
    loss = -(logp.mean() + gamma * entropy.mean()).item()
    dlogits = Q.qadc_token_logprobs_backward(logits, tokens, lse, entropy, torch.full_like(logp, -1.0 / rows),
                                             torch.full_like(entropy, -gamma / rows))
    dstate = (dlogits.float() @ head).bfloat16()
    _, dweight, dbias = Q.qadc_layer_norm_backward(dstate, hidden, weight, mean, rstd, need_dx=False)
    weight -= rate * dweight
    bias -= rate * dbias
    return loss


def main(states=200_000, batch=32, steps=40, seed=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    prototypes, head, scale, offset = make_model(g)
    hidden, values = observe(prototypes, scale, offset, states, g)

    weight, bias = torch.ones((D,), device=DEV), torch.zeros((D,), device=DEV)
    losses = []
    for step in range(steps):
        at = torch.randint(0, states, (2048,), generator=g, device=DEV)
        losses.append(train_step(hidden[at].contiguous(), values[at].contiguous(), weight, bias, head, 1.0))
    if steps:
        print(f"training the norm: loss {losses[0]:.3f} -> {losses[-1]:.3f} in {steps} steps")

    normed, _, _ = Q.qadc_layer_norm(hidden, weight, bias)
    codebooks, codes = build_datastore(normed.float())
    packed = quantize_head(head)
    queries, targets = observe(prototypes, scale, offset, 512, g)
    own, mixed = score(queries, targets, weight, bias, packed, codebooks, codes, values)
    print(f"{states} stored states: -log p of what followed {own:.3f} by the model alone, {mixed:.3f} with its neighbours")

    candidates, mix, _ = decode(queries[:batch].contiguous(), weight, bias, packed, codebooks, codes, values)
    choice = torch.gather(candidates, 1, mix.argmax(1, keepdim=True))[:, 0]
    right = (choice == targets[:batch]).float().mean().item()
    print(f"a decode step of {batch} sequences: {100 * right:.0f} % of the tokens right")
    return {"losses": losses, "own": own, "mixed": mixed, "right": right}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--states", type=int, default=200_000)
    ap.add_argument("--batch", type=int, default=32)
    ap.add_argument("--steps", type=int, default=40)
    a = ap.parse_args()
    main(a.states, a.batch, a.steps)
