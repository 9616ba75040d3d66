"""The language-model operators next to the search, as cases that can be timed and compared.

A decode step over a datastore of hidden states normalises the state (`norm`), multiplies it with
4-bit weights up to the vocabulary's logits (`linear4`), takes the log probabilities of the tokens
of interest and the likeliest alternatives (`logprobs`), and mixes in the tokens that followed the
nearest stored states (`mix`). Training the encoder runs the norm and the log probabilities
backwards (`norm_grad`, `logprobs_grad`).

Where `own` is false `run` computes an operator in its plain form: elementary torch operations in
float32, rounded once at the end. Where it is true, it calls the library.
"""

import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-5

# Ranges, and the largest number of elements (or weights) that a drawn case takes.
MAX_NORM = 16384 * 4096
MAX_WEIGHTS = 131072 * 4096
MAX_LOGITS = 4096 * 65536
MAX_VOTES = 2048 * 1024
DEV = "cuda:0"


# ---------------------------------------------------------------------------------------------
# cases

def _norm(rows, d, type, grad):
    return {"kind": "norm_grad" if grad else "norm", "rows": rows, "d": d, "type": type}


def _linear4(M, N, K, group, type, zeros):
    return {"kind": "linear4", "M": M, "N": N, "K": K, "group": group, "type": type, "zeros": zeros}


def _logprobs(rows, V, T, k, type, scale=1.0, masked=False):
    return {"kind": "logprobs", "rows": rows, "V": V, "T": T, "k": k, "type": type, "scale": scale, "masked": masked}


def _logprobs_grad(rows, V, T, type, scale=1.0, entropy=True):
    return {"kind": "logprobs_grad", "rows": rows, "V": V, "T": T, "type": type, "scale": scale, "entropy": entropy}


def _mix(rows, R, T, n, dist):
    return {"kind": "mix", "rows": rows, "R": R, "T": T, "n": n, "dist": dist}


def listed():
    return [
        # the hidden states of a decode step of five sequences: a call is all latency
        dict(_norm(5, 4096, "bf16", False), name="norm_decode"),
        # the backward pass of one training step of an encoder: 16384 tokens
        dict(_norm(16384, 4096, "bf16", True), name="norm_grad_train"),
        # the same of a small embedding model in float32, with an odd width and a ragged batch
        dict(_norm(2049, 1111, "f32", True), name="norm_grad_odd"),
        # one token through a square projection
        dict(_linear4(1, 4096, 4096, 128, "f16", False), name="linear4_token"),
        # one token through the vocabulary head, the largest matrix of a decode step
        dict(_linear4(1, 131072, 4096, 128, "bf16", False), name="linear4_head"),
        # a batch of 24 sequences through weights with fine groups and zero points, sizes that fill no tile
        dict(_linear4(24, 10007, 5000, 32, "bf16", True), name="linear4_batch"),
        # one token's logits: its log probability and 20 alternatives
        dict(_logprobs(1, 131072, 1, 20, "bf16"), name="logprobs_token"),
        # a batch under constrained decoding: the tokens that the neighbours vote for, 50 alternatives
        dict(_logprobs(64, 50021, 100, 50, "f16", 1.25, True), name="logprobs_batch"),
        # scoring the tokens of a training step, float16/32 masters aside: only the log probabilities and the entropy
        dict(_logprobs(4096, 65536, 1, 0, "bf16"), name="logprobs_score"),
        # and the gradient of that step
        dict(_logprobs_grad(4096, 65536, 1, "bf16"), name="logprobs_grad_train"),
        # one token's mixture: the neighbours of one search of 10 M codes, quantized sums
        dict(_mix(1, 100, 120, 10_000_000, "u8"), name="mix_token"),
        # evaluation of 2048 tokens, the most neighbours that a search returns, float distances
        dict(_mix(2048, 1024, 64, 10_000_000, "f32"), name="mix_eval"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "linear4", "linear4", "logprobs", "logprobs", "logprobs_grad", "mix"])
    type = rng.choice(["f32", "f16", "bf16"])
    if kind in ("norm", "norm_grad"):
        d = _log(rng, 64, 16384)
        return _norm(_log(rng, 1, min(16384, MAX_NORM // (d * BYTES[type] // 2))), d, type, kind == "norm_grad")
    if kind == "linear4":
        K = _log(rng, 256, 16384)
        N = _log(rng, 256, min(131072, MAX_WEIGHTS // K))
        M = _log(rng, 1, max(1, min(64, MAX_WEIGHTS // (K * N) * 4)))
        return _linear4(M, N, K, rng.choice([32, 64, 128]), type, rng.random() < 0.5)
    if kind == "logprobs":
        V = _log(rng, 1000, 262144)
        rows = _log(rng, 1, min(4096, MAX_LOGITS // (V * BYTES[type] // 2)))
        return _logprobs(rows, V, _log(rng, 1, 128), rng.choice([0, 1, _log(rng, 2, 64)]), type,
                         rng.choice([1.0, round(rng.uniform(0.5, 2.0), 3)]), rng.random() < 0.3)
    if kind == "logprobs_grad":
        V = _log(rng, 1000, 262144)
        rows = _log(rng, 1, min(4096, MAX_LOGITS // (V * BYTES[type] // 2)))
        return _logprobs_grad(rows, V, rng.choice([1, _log(rng, 1, 16)]), type,
                              rng.choice([1.0, round(rng.uniform(0.5, 2.0), 3)]), rng.random() < 0.5)
    R = _log(rng, 1, 1024)
    rows = _log(rng, 1, MAX_VOTES // 1024)
    return _mix(rows, R, _log(rng, 1, 128), _log(rng, 10_000, 20_000_000), rng.choice(["u8", "f32"]))


# ---------------------------------------------------------------------------------------------
# inputs

def _logits(rows, V, type, g, masked=False):
    """Logits as a model gives them: a wide bulk, and in each row a few dozen tokens well above it. Under constrained decoding
    (`masked`) a grammar leaves a share of the tokens, in every eighth row only one in fifty."""
    x = torch.randn((rows, V), generator=g, device=DEV).mul_(2.0)
    top = torch.randint(0, V, (rows, 32), generator=g, device=DEV)
    x.scatter_add_(1, top, 4.0 + 3.0 * torch.rand((rows, 32), generator=g, device=DEV))
    if masked:
        share = torch.full((rows, 1), 0.7, device=DEV)
        share[::8] = 0.02
        x.masked_fill_(torch.rand((rows, V), generator=g, device=DEV) >= share, -math.inf)
    return x.to(TYPES[type])


def _states(rows, d, type, g):
    """Hidden states: every row with its own offset and spread, a few outlying columns."""
    x = torch.randn((rows, d), generator=g, device=DEV)
    x = x * (0.5 + torch.rand((rows, 1), generator=g, device=DEV)) + 0.3 * torch.randn((rows, 1), generator=g, device=DEV)
    at = torch.randint(0, d, (max(1, d // 256),), generator=g, device=DEV)
    x[:, at] *= 12.0
    return x.to(TYPES[type])


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    c = dict(case)
    kind = c["kind"]
    if kind in ("norm", "norm_grad"):
        c["x"] = _states(c["rows"], c["d"], c["type"], g)
        c["w"] = 1.0 + 0.1 * torch.randn((c["d"],), generator=g, device=DEV)
        c["b"] = 0.1 * torch.randn((c["d"],), generator=g, device=DEV)
        if kind == "norm_grad":
            c["dy"] = (0.01 * torch.randn((c["rows"], c["d"]), generator=g, device=DEV)).to(TYPES[c["type"]])
            x = c["x"].float()
            c["mean"] = x.mean(1)
            c["rstd"] = torch.rsqrt(x.var(1, correction=0) + EPS)
            if own:  # the scratch memory that a training program keeps
                import paper_1704_07355_amd as Q
                c["ws"] = torch.empty((Q.qadc_layer_norm_workspace_bytes(c["rows"], c["d"]),), dtype=torch.uint8, device=DEV)
    elif kind == "linear4":
        M, N, K, G = c["M"], c["N"], c["K"], c["group"]
        c["x"] = _states(M, K, c["type"], g)
        groups = -(-K // G)
        # codes of nearly normal weights around the zero point: byte j holds element 2j low and element 2j + 1 high
        wide = [torch.randn((N, -(-K // 2)), generator=g, device=DEV).mul_(2.6).add_(8.0).round_().clamp_(0, 15).to(torch.uint8)
                for _ in range(2)]
        c["codes"] = wide[0] | (wide[1] << 4)
        del wide
        c["scales"] = (0.004 + 0.008 * torch.rand((N, groups), generator=g, device=DEV)).to(
            torch.bfloat16 if c["type"] == "bf16" else torch.float16)
        c["zeros"] = (torch.randint(5, 12, (N, groups), generator=g, device=DEV, dtype=torch.uint8) if c["zeros"] else None)
        if own:  # the weights as a serving program keeps them
            import paper_1704_07355_amd as Q
            c["weights"] = Q.qadc_pack_weights4(c["codes"], c["scales"], c["zeros"], K, G)
    elif kind in ("logprobs", "logprobs_grad"):
        rows, V, T = c["rows"], c["V"], c["T"]
        c["logits"] = _logits(rows, V, c["type"], g, c.get("masked", False))
        c["tokens"] = torch.randint(0, V, (rows, T), generator=g, device=DEV, dtype=torch.int32)
        # sequences end at their own lengths: one in sixteen slots is unused
        c["tokens"][torch.rand((rows, T), generator=g, device=DEV) < 1 / 16] = -1
        if kind == "logprobs_grad":
            x = c["logits"].float() * c["scale"]
            c["lse"] = torch.logsumexp(x, 1)
            p = torch.exp(x - c["lse"][:, None])
            c["H"] = c["lse"] - (p * x).sum(1)
            del x, p
            c["dlogp"] = torch.randn((rows, T), generator=g, device=DEV)
            c["dH"] = 0.1 * torch.randn((rows,), generator=g, device=DEV) if c["entropy"] else None
        elif own:
            import paper_1704_07355_amd as Q
            c["ws"] = Q.qadc_workspace_init(torch.empty(
                (max(256, Q.qadc_token_logprobs_workspace_bytes(rows, V, c["k"])),), dtype=torch.uint8, device=DEV))
    else:
        rows, R, T, n = c["rows"], c["R"], c["T"], c["n"]
        V = 32768
        # tokens follow each other unevenly: the square of a uniform number
        u = torch.rand((n,), generator=g, device=DEV)
        c["values"] = (u * u * V).to(torch.int32).clamp_(max=V - 1)
        c["ids"] = torch.randint(0, n, (rows, R), generator=g, device=DEV, dtype=torch.int32)
        c["ids"][:, R - R // 16:] = -1  # a short list's padding: 0xFFFFFFFF
        if c["dist"] == "u8":
            c["d"] = torch.sort(torch.randint(40, 256, (rows, R), generator=g, device=DEV, dtype=torch.uint8), dim=1).values
            c["step"] = 150.0 + 100.0 * torch.rand((rows,), generator=g, device=DEV)
        else:
            c["d"] = torch.sort(8000.0 + 40000.0 * torch.rand((rows, R), generator=g, device=DEV), dim=1).values
            c["step"] = None
        c["beta"], c["lam"] = 1 / 4000.0, 0.25
        # the tokens of interest: some that neighbours vote for, the others of the model's own choice
        own_choice = torch.randint(0, V, (rows, T), generator=g, device=DEV, dtype=torch.int32)
        at = torch.randint(0, max(1, R - R // 16), (rows, T), generator=g, device=DEV)
        voted = c["values"][torch.gather(c["ids"], 1, at).clamp(min=0).long()]
        c["tokens"] = torch.where(torch.rand((rows, T), generator=g, device=DEV) < 0.5, voted, own_choice).contiguous()
        c["tokens"][torch.rand((rows, T), generator=g, device=DEV) < 1 / 32] = -1
        c["lm"] = -12.0 * torch.rand((rows, T), generator=g, device=DEV)
    return c


# ---------------------------------------------------------------------------------------------
# one pass

def _unpack4(codes, K):
    q = torch.stack((codes & 15, codes >> 4), dim=-1).reshape(codes.shape[0], -1)
    return q[:, :K]


def _plain_norm(c):
    x = c["x"].float()
    mean = x.mean(1)
    h = x - mean[:, None]
    rstd = torch.rsqrt((h * h).mean(1) + EPS)
    return {"y": (h * rstd[:, None] * c["w"] + c["b"]).to(c["x"].dtype), "mean": mean, "rstd": rstd}


def _plain_norm_grad(c):
    dy = c["dy"].float()
    h = (c["x"].float() - c["mean"][:, None]) * c["rstd"][:, None]
    g = dy * c["w"]
    dx = (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True)) * c["rstd"][:, None]
    return {"dx": dx.to(c["x"].dtype), "dw": (dy * h).sum(0), "db": dy.sum(0)}


def _plain_linear4(c):
    q = _unpack4(c["codes"], c["K"]).float()
    of = torch.arange(c["K"], device=DEV) // c["group"]
    zero = 8.0 if c["zeros"] is None else c["zeros"].float()[:, of]
    w = (q - zero) * c["scales"].float()[:, of]
    return {"y": (c["x"].float() @ w.t()).to(c["x"].dtype)}


def _plain_logprobs(c):
    logits, V, k = c["logits"].float(), c["V"], c["k"]
    x = logits * c["scale"]
    m = x.max(1, keepdim=True).values
    e = torch.exp(x - m)
    s = e.sum(1)
    lse = m[:, 0] + torch.log(s)
    H = torch.log(s) - torch.where(e > 0, e * (x - m), 0.0).sum(1) / s
    used = (c["tokens"] >= 0) & (c["tokens"] < V)
    at = torch.where(used, c["tokens"], 0).long()
    out = {"logp": torch.where(used, torch.gather(x, 1, at) - lse[:, None], 0.0), "lse": lse, "H": H}
    if k:
        # the order (logit descending, index ascending) as one whole number: the float's bits made monotone, then the index
        bits = (logits + 0.0).view(torch.int32).long()
        up = torch.where(bits < 0, -2147483648 - bits - 1, bits)
        key = (up << 32) + (V - 1 - torch.arange(V, device=DEV))
        idx = V - 1 - (torch.topk(key, k, dim=1).values & 0xFFFFFFFF)
        out["top"] = idx.to(torch.int32)
        out["top_logp"] = torch.gather(x, 1, idx) - lse[:, None]
    return out


def _plain_logprobs_grad(c):
    x = c["logits"].float() * c["scale"]
    lp = x - c["lse"][:, None]
    p = torch.exp(lp)
    used = (c["tokens"] >= 0) & (c["tokens"] < c["V"])
    dl = torch.where(used, c["dlogp"], 0.0)
    dx = -dl.sum(1, keepdim=True) * p
    if c["dH"] is not None:
        dx -= c["dH"][:, None] * torch.where(p > 0, p * (lp + c["H"][:, None]), 0.0)
    dx.scatter_add_(1, torch.where(used, c["tokens"], 0).long(), dl)
    return {"dlogits": (dx * c["scale"]).to(c["logits"].dtype)}


def _plain_mix(c):
    used = c["ids"] >= 0
    value = torch.where(used, c["values"][c["ids"].clamp(min=0).long()], -1)
    dist = c["d"].float()
    near = torch.where(used, dist, math.inf).min(1, keepdim=True).values
    v = -(dist - near) * c["beta"]
    if c["step"] is not None:
        v = v * c["step"][:, None]
    v = torch.where(used, v, -math.inf)
    w = torch.exp(v - torch.logsumexp(v, 1, keepdim=True))
    w = torch.where(used.any(1, keepdim=True), w, 0.0)
    tok = c["tokens"]
    votes = (w[:, None, :] * (value[:, None, :] == tok[:, :, None])).sum(2)
    knn = torch.log(votes)
    lam = torch.where(used.any(1, keepdim=True), c["lam"], 0.0)
    mix = torch.logaddexp(c["lm"] + torch.log1p(-lam), knn + torch.log(lam))
    return {"mix": torch.where(tok >= 0, mix, 0.0), "knn": torch.where(tok >= 0, knn, 0.0)}


PLAIN = {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "linear4": _plain_linear4, "logprobs": _plain_logprobs,
         "logprobs_grad": _plain_logprobs_grad, "mix": _plain_mix}


def run(state):
    c = state
    if not own:
        return PLAIN[c["kind"]](c)
    import paper_1704_07355_amd as Q
    if c["kind"] == "norm":
        y, mean, rstd = Q.qadc_layer_norm(c["x"], c["w"], c["b"], EPS)
        return {"y": y, "mean": mean, "rstd": rstd}
    if c["kind"] == "norm_grad":
        dx, dw, db = Q.qadc_layer_norm_backward(c["dy"], c["x"], c["w"], c["mean"], c["rstd"], workspace=c["ws"])
        return {"dx": dx, "dw": dw, "db": db}
    if c["kind"] == "linear4":
        return {"y": Q.qadc_linear4(c["weights"], c["x"])}
    if c["kind"] == "logprobs":
        logp, lse, H, top, top_logp = Q.qadc_token_logprobs(c["logits"], c["tokens"], c["k"], c["scale"], workspace=c["ws"])
        out = {"logp": logp, "lse": lse, "H": H}
        if c["k"]:
            out["top"], out["top_logp"] = top, top_logp
        return out
    if c["kind"] == "logprobs_grad":
        return {"dlogits": Q.qadc_token_logprobs_backward(c["logits"], c["tokens"], c["lse"], c["H"], c["dlogp"], c["dH"],
                                                          c["scale"])}
    mix, knn = Q.qadc_neighbour_mix(c["ids"], c["d"], c["values"], c["tokens"], c["lm"], c["lam"], c["beta"], c["step"])
    return {"mix": mix, "knn": knn}


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without

def work(case):
    c, kind = case, case["kind"]
    e = BYTES[c["type"]] if "type" in c else 0
    if kind == "norm":
        n = c["rows"] * c["d"]
        return {"bytes": 2 * n * e + 8 * c["rows"] + 8 * c["d"], "flops": 8 * n}
    if kind == "norm_grad":
        n = c["rows"] * c["d"]
        return {"bytes": 3 * n * e + 8 * c["rows"] + 12 * c["d"], "flops": 14 * n}
    if kind == "linear4":
        M, N, K = c["M"], c["N"], c["K"]
        groups = -(-K // c["group"])
        return {"bytes": N * -(-K // 2) + N * groups * (3 if c["zeros"] else 2) + M * (K + N) * e, "flops": 2 * M * N * K}
    if kind == "logprobs":
        n = c["rows"] * c["V"]
        return {"bytes": n * e + c["rows"] * (8 * c["T"] + 8 * c["k"] + 8), "flops": 6 * n}
    if kind == "logprobs_grad":
        n = c["rows"] * c["V"]
        return {"bytes": 2 * n * e + c["rows"] * (8 * c["T"] + 12), "flops": 6 * n}
    votes = c["rows"] * c["R"]
    return {"bytes": votes * (8 + (1 if c["dist"] == "u8" else 4)) + c["rows"] * c["T"] * 16, "flops": 4 * votes}


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits

def exact(case, seed):
    c = prepare(case, seed)
    kind = c["kind"]
    if kind == "norm":
        x = c["x"].double()
        mean = torch.sum(x, 1) / c["d"]
        var = torch.sum((x - mean[:, None]) ** 2, 1) / c["d"]
        rstd = 1 / torch.sqrt(var + EPS)
        return {"y": (x - mean[:, None]) * rstd[:, None] * c["w"].double() + c["b"].double(), "mean": mean, "rstd": rstd}
    if kind == "norm_grad":
        x, dy, w = c["x"].double(), c["dy"].double(), c["w"].double()
        mean, rstd = c["mean"].double()[:, None], c["rstd"].double()[:, None]
        xhat = (x - mean) * rstd
        a = torch.sum(dy * w, 1, keepdim=True) / c["d"]
        b = torch.sum(dy * w * xhat, 1, keepdim=True) / c["d"]
        return {"dx": rstd * (dy * w - a - xhat * b), "dw": torch.sum(dy * xhat, 0), "db": torch.sum(dy, 0)}
    if kind == "linear4":
        x, N, K, G = c["x"].double(), c["N"], c["K"], c["group"]
        y = torch.empty((c["M"], N), dtype=torch.float64, device=DEV)
        for r in range(0, N, 8192):
            part = c["codes"][r:r + 8192].long()
            w = torch.empty((part.shape[0], 2 * part.shape[1]), dtype=torch.float64, device=DEV)
            w[:, 0::2], w[:, 1::2] = (part % 16).double(), (part // 16).double()
            w = w[:, :K]
            for k in range(0, K, G):
                z = 8.0 if c["zeros"] is None else c["zeros"][r:r + 8192, k // G, None].double()
                w[:, k:k + G] = (w[:, k:k + G] - z) * c["scales"][r:r + 8192, k // G, None].double()
            y[:, r:r + 8192] = torch.mm(x, w.t().contiguous())
        return {"y": y}
    if kind in ("logprobs", "logprobs_grad"):
        rows, V = c["rows"], c["V"]
        parts = []
        for r in range(0, rows, 512):
            x = c["logits"][r:r + 512].double() * c["scale"]
            tok = c["tokens"][r:r + 512].long()
            off = (tok < 0) | (tok >= V)
            tok = tok.masked_fill(off, 0)
            if kind == "logprobs":
                lp = torch.log_softmax(x, 1)
                some = torch.isfinite(x)
                part = {"logp": torch.gather(lp, 1, tok).masked_fill(off, 0.0), "lse": torch.logsumexp(x, 1),
                        "H": -torch.sum(torch.exp(lp) * lp.masked_fill(~some, 0.0), 1)}
                if c["k"]:
                    part["top_logp"] = torch.sort(lp, dim=1, descending=True).values[:, :c["k"]].clone()
            else:
                lp = x - c["lse"][r:r + 512, None].double()
                d = c["dlogp"][r:r + 512].double().masked_fill(off, 0.0)
                dx = torch.zeros_like(x).scatter_add(1, tok, d) - torch.exp(lp) * torch.sum(d, 1, keepdim=True)
                if c["dH"] is not None:
                    dx = dx - c["dH"][r:r + 512, None].double() * torch.exp(lp) * (lp + c["H"][r:r + 512, None].double())
                part = {"dlogits": dx * c["scale"]}
            parts.append(part)
        out = {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
        if c.get("k"):
            out["top"] = None
        return out
    used = c["ids"] >= 0
    value = c["values"][c["ids"].clamp(min=0).long()].masked_fill(~used, -7)
    v = -c["d"].double() * c["beta"] * (1.0 if c["step"] is None else c["step"].double()[:, None])
    w = torch.softmax(v.masked_fill(~used, -math.inf), 1)
    votes = torch.stack([torch.sum(w * (value == c["tokens"][:, t, None]), 1) for t in range(c["T"])], 1)
    mix = torch.log((1 - c["lam"]) * torch.exp(c["lm"].double()) + c["lam"] * votes)
    off = c["tokens"] < 0
    return {"mix": mix.masked_fill(off, 0.0), "knn": torch.log(votes).masked_fill(off, 0.0)}
