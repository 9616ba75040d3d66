"""More language-model operators next to the search, as cases that can be timed and compared.

A decode step adds the residual and normalises it by its root mean square, in 8 bits where the products that follow take them
(`rms`); beside the shared projection each request has its own low-rank adapter (`adapters`); the logits that come out are
penalised, biased and masked (`adjust`) before their log probabilities are taken. Training runs the norm backwards (`rms_grad`)
and distils a teacher whose likeliest tokens were stored: the loss (`distill`), its gradient (`distill_grad`), or both in one call
(`distill_step`).

Where `own` is false `run` computes an operator in its plain form: elementary torch operations in
float32, rounded once at the end. Where it is true, it calls the library.
"""

import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-5
E4M3_MAX = 448.0

# The most elements (of 16 bits) that a drawn case takes: rows of states, logits that are adjusted, logits of a loss; for adapters
# the rows' elements and those of all adapters.
MAX_NORM = 16384 * 4096
MAX_ADJUST = 256 * 131072
MAX_LOGITS = 4096 * 65536
MAX_ROWS, MAX_ADAPTERS = 8192 * 8192, 16 * 64 * 8192
DEV = "cuda:0"


# ---------------------------------------------------------------------------------------------
# cases

def _rms(rows, d, type, residual, e4m3):
    return {"kind": "rms", "rows": rows, "d": d, "type": type, "residual": residual, "e4m3": e4m3}


def _rms_grad(rows, d, type, residual):
    return {"kind": "rms_grad", "rows": rows, "d": d, "type": type, "residual": residual}


def _adjust(rows, V, H, B, type, masked):
    return {"kind": "adjust", "rows": rows, "V": V, "H": H, "B": B, "type": type, "masked": masked}


def _distill(kind, rows, V, k, type, scale, tail):
    return {"kind": kind, "rows": rows, "V": V, "k": k, "type": type, "scale": scale, "tail": tail}


def _adapters(M, N, K, rank, count, type, segments):
    return {"kind": "adapters", "M": M, "N": N, "K": K, "rank": rank, "count": count, "type": type, "segments": segments}


def listed():
    return [
        # the states of a decode step of five sequences, the residual added, in 8 bits for the products that follow
        dict(_rms(5, 4096, "bf16", True, True), name="rms_decode"),
        # the backward pass of one training step: 16384 tokens, with the gradient that comes down the residual
        dict(_rms_grad(16384, 4096, "bf16", True), name="rms_grad_train"),
        # the same of a small model in float32, with an odd width and a ragged batch, of a norm without a residual
        dict(_rms_grad(3001, 1537, "f32", False), name="rms_grad_odd"),
        # one sequence's logits: 2048 tokens of history, a few biases, a grammar
        dict(_adjust(1, 131072, 2048, 16, "bf16", True), name="adjust_token"),
        # a batch of sequences with long histories, a grammar for some of them, a vocabulary that fills no pack
        dict(_adjust(256, 128001, 4099, 32, "f16", True), name="adjust_batch"),
        # the loss of a few sequences' answers at a higher temperature, without the tail
        dict(_distill("distill", 48, 50021, 50, "f16", 0.5, False), name="distill_few"),
        # the gradient alone, float32 logits of a small vocabulary
        dict(_distill("distill_grad", 1111, 32003, 20, "f32", 1.0, True), name="distill_grad_odd"),
        # a training step: loss and gradient of 4096 tokens with 64 stored logits each
        dict(_distill("distill_step", 4096, 65536, 64, "bf16", 1.0, True), name="distill_step_train"),
        # the same of a large vocabulary whose rows begin anywhere
        dict(_distill("distill_step", 512, 128001, 100, "bf16", 1.0, True), name="distill_step_odd"),
        # one token through a square projection
        dict(_adapters(1, 4096, 4096, 16, 8, "f16", False), name="adapters_token"),
        # a batch of 64 sequences, each with one of 32 adapters, beside a wide projection
        dict(_adapters(64, 16384, 4096, 16, 32, "bf16", False), name="adapters_batch"),
        # the prompts of 16 requests, 8192 tokens together
        dict(_adapters(8192, 4096, 4096, 64, 16, "bf16", True), name="adapters_prompt"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(["rms", "rms_grad", "adjust", "adjust", "distill", "distill_grad", "distill_step", "adapters", "adapters", "adapters"])
    type = rng.choice(["f32", "f16", "bf16"])
    wide = BYTES[type] // 2
    if kind in ("rms", "rms_grad"):
        d = _log(rng, 64, 16384)
        rows = _log(rng, 1, min(16384, MAX_NORM // (d * wide)))
        return _rms(rows, d, type, rng.random() < 0.7, rng.random() < 0.5) if kind == "rms" else _rms_grad(rows, d, type, rng.random() < 0.7)
    if kind == "adjust":
        V = _log(rng, 1000, 262144)
        return _adjust(_log(rng, 1, min(1024, MAX_ADJUST // (V * wide))), V, _log(rng, 1, 32768),
                       rng.choice([0, _log(rng, 1, 512)]), type, rng.random() < 0.5)
    if kind == "adapters":
        rank, count = rng.choice([8, 16, 32, 64, _log(rng, 1, 128)]), _log(rng, 1, 64)
        most = max(1024, MAX_ADAPTERS // (rank * count * wide))
        K = _log(rng, 256, min(16384, most - 256))
        N = _log(rng, 256, min(16384, most - K)) if most - K > 256 else 256
        return _adapters(_log(rng, 1, min(8192, MAX_ROWS // ((K + N) * wide))), N, K, rank, count, type, rng.random() < 0.5)
    V = _log(rng, 1000, 262144)
    return _distill(kind, _log(rng, 1, min(4096, MAX_LOGITS // (V * wide))), V, rng.choice([1, _log(rng, 2, 128), _log(rng, 2, 128)]),
                    type, rng.choice([1.0, round(rng.uniform(0.25, 1.5), 3)]), rng.random() < 0.7)


# ---------------------------------------------------------------------------------------------
# inputs

def _logits(rows, V, type, g):
    """Logits as a model gives them: a wide bulk, and in each row a few dozen tokens well above it."""
    x = torch.randn((rows, V), generator=g, device=DEV).mul_(2.0)
    top = torch.randint(0, V, (rows, 32), generator=g, device=DEV)
    return x.scatter_add_(1, top, 4.0 + 3.0 * torch.rand((rows, 32), generator=g, device=DEV)).to(TYPES[type])


def _states(rows, d, type, g):
    """Hidden states: every row with its own spread, a few outlying columns."""
    x = torch.randn((rows, d), generator=g, device=DEV) * (0.5 + torch.rand((rows, 1), generator=g, device=DEV))
    at = torch.randint(0, d, (max(1, d // 256),), generator=g, device=DEV)
    x[:, at] *= 12.0
    return x.to(TYPES[type])


def _ranks(c):
    """Every third adapter has about half the ranks that the pool has room for."""
    return [c["rank"] if a % 3 < 2 else (c["rank"] + 1) // 2 for a in range(c["count"])]


def _rows_without(M):
    """Rows of a mixed batch that have no adapter: one in thirteen."""
    return M // 13


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    c = dict(case)
    kind = c["kind"]
    if kind in ("rms", "rms_grad"):
        rows, d = c["rows"], c["d"]
        c["x"] = _states(rows, d, c["type"], g)
        c["w"] = 1.0 + 0.1 * torch.randn((d,), generator=g, device=DEV)
        if kind == "rms":
            c["res"] = _states(rows, d, c["type"], g) if c["residual"] else None
        else:
            c["dy"] = (0.01 * torch.randn((rows, d), generator=g, device=DEV)).to(TYPES[c["type"]])
            c["dsum"] = (0.01 * torch.randn((rows, d), generator=g, device=DEV)).to(TYPES[c["type"]]) if c["residual"] else None
            c["rstd"] = torch.rsqrt(c["x"].float().square().mean(1) + EPS)
            if own:  # the scratch memory that a training program keeps
                import paper_1704_07355_amd as Q
                c["ws"] = torch.empty((Q.qadc_rms_norm_workspace_bytes(rows, d),), dtype=torch.uint8, device=DEV)
    elif kind == "adjust":
        rows, V, H, B = c["rows"], c["V"], c["H"], c["B"]
        c["logits"] = _logits(rows, V, c["type"], g)
        c["bias_tokens"] = c["bias"] = c["masks"] = c["mask_of"] = None
        # tokens follow each other unevenly; sequences have their own lengths and settings
        u = torch.rand((rows, H), generator=g, device=DEV)
        c["history"] = (u * u * u * V).to(torch.int32).clamp_(max=V - 1)
        c["lengths"] = torch.randint(H // 2, H + 1, (rows,), generator=g, device=DEV, dtype=torch.int32)
        c["prompt"] = c["lengths"] // 3
        c["rep"] = 1.0 + 0.3 * torch.rand((rows,), generator=g, device=DEV)
        c["freq"] = 0.2 * torch.rand((rows,), generator=g, device=DEV)
        c["pres"] = 0.5 * torch.rand((rows,), generator=g, device=DEV)
        if B:
            c["bias_tokens"] = torch.randint(0, V, (rows, B), generator=g, device=DEV, dtype=torch.int32)
            c["bias_tokens"][torch.rand((rows, B), generator=g, device=DEV) < 1 / 8] = -1  # unused slots
            c["bias"] = 3.0 * torch.randn((rows, B), generator=g, device=DEV)
        if c["masked"]:  # the grammar's states: bit v % 32 of word v / 32. Every third sequence has none
            states, words = min(rows, 64), -(-V // 32)
            share = torch.full((states, 1, 1), 0.7, device=DEV)
            share[::2] = 0.02
            bits = (torch.rand((states, words, 32), generator=g, device=DEV) < share).long()
            packed = (bits << torch.arange(32, device=DEV)).sum(2)
            c["masks"] = torch.where(packed >= 1 << 31, packed - (1 << 32), packed).to(torch.int32)
            c["mask_of"] = torch.randint(0, states, (rows,), generator=g, device=DEV, dtype=torch.int32)
            c["mask_of"][2::3] = -1
    elif kind == "adapters":
        M, N, K, r, n = c["M"], c["N"], c["K"], c["rank"], c["count"]
        t = TYPES[c["type"]]
        c["x"] = _states(M, K, c["type"], g)
        c["base"] = torch.randn((M, N), generator=g, device=DEV).to(t)
        c["a"] = (torch.randn((n, r, K), generator=g, device=DEV) / math.sqrt(K)).to(t)
        c["b"] = (0.2 * torch.randn((n, N, r), generator=g, device=DEV)).to(t)
        c["scales"] = 0.5 + torch.rand((n,), generator=g, device=DEV)
        c["ranks"] = torch.tensor(_ranks(c), dtype=torch.int32, device=DEV)
        if c["segments"]:  # requests of about the same length, one after the other
            c["ids"] = (torch.arange(M, device=DEV) * n // M).to(torch.int32)
        else:
            some = M - _rows_without(M)
            ids = torch.cat((torch.arange(some, device=DEV) % n, torch.full((M - some,), -1, device=DEV)))
            c["ids"] = ids[torch.randperm(M, generator=g, device=DEV)].to(torch.int32)
        if own:
            import paper_1704_07355_amd as Q
            c["adapters"] = Q.qadc_adapters(c["a"], c["b"], c["scales"], c["ranks"])
            c["ws"] = torch.empty((max(256, Q.qadc_adapters_workspace_bytes(c["adapters"], M)),), dtype=torch.uint8, device=DEV)
    else:
        rows, V, k = c["rows"], c["V"], c["k"]
        c["logits"] = _logits(rows, V, c["type"], g)
        # the teacher agrees with the student up to noise; the stored logits of some rows are fewer
        c["top"] = torch.empty((rows, k), dtype=torch.int32, device=DEV)
        c["top_logp"] = torch.empty((rows, k), device=DEV)
        for r in range(0, rows, 1024):
            t = c["logits"][r:r + 1024].float() * c["scale"]
            t += 0.5 * torch.randn(t.shape, generator=g, device=DEV)
            lp, at = torch.topk(t, k, dim=1)
            c["top"][r:r + 1024], c["top_logp"][r:r + 1024] = at.to(torch.int32), lp - torch.logsumexp(t, 1, keepdim=True)
        del t
        if k > 8:
            c["top"][::4, k - k // 8:], c["top_logp"][::4, k - k // 8:] = -1, -math.inf
        # a row's share of the loss: one of sixteen belongs to a prompt and has none
        c["weight"] = torch.where(torch.rand((rows,), generator=g, device=DEV) < 1 / 16, 0.0, 0.5 + torch.rand((rows,), generator=g, device=DEV))
        if kind == "distill_grad":
            lse, log_tail = [], []
            for r in range(0, rows, 1024):
                x = c["logits"][r:r + 1024].float() * c["scale"]
                lse.append(torch.logsumexp(x, 1))
                at = c["top"][r:r + 1024]
                x = torch.cat((x, x[:, :1]), 1).scatter_(1, torch.where(at >= 0, at, V).long(), -math.inf)
                x[:, V] = -math.inf
                log_tail.append(torch.logsumexp(x, 1) - lse[-1])
            c["lse"], c["log_tail"] = torch.cat(lse), torch.cat(log_tail)
        elif own:
            import paper_1704_07355_amd as Q
            c["ws"] = torch.empty((max(256, Q.qadc_distill_workspace_bytes(rows, V)),), dtype=torch.uint8, device=DEV)
    return c


# ---------------------------------------------------------------------------------------------
# one pass

def _plain_rms(c):
    type, x = c["x"].dtype, c["x"].float()
    out = {}
    if c["res"] is not None:
        out["sum"] = (x + c["res"].float()).to(type)
        x = out["sum"].float()
    out["rstd"] = torch.rsqrt((x * x).mean(1) + EPS)
    y = x * out["rstd"][:, None] * c["w"]
    if not c["e4m3"]:
        return dict(out, y=y.to(type))
    most = y.abs().amax(1)
    return dict(out, y=(y * (E4M3_MAX / most)[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), scale=most / E4M3_MAX)


def _plain_rms_grad(c):
    dy, rstd = c["dy"].float(), c["rstd"][:, None]
    h = c["x"].float() * rstd
    g = dy * c["w"]
    dx = rstd * (g - h * (g * h).mean(1, keepdim=True))
    if c["dsum"] is not None:
        dx = dx + c["dsum"].float()
    return {"dx": dx.to(c["x"].dtype), "dw": (dy * h).sum(0)}


def _plain_adjust(c):
    rows, V = c["rows"], c["V"]
    x = c["logits"].float()
    at, h = torch.arange(c["H"], device=DEV), c["history"].long()
    there = at < c["lengths"][:, None]
    said = (there & (at >= c["prompt"][:, None])).float()
    seen = torch.zeros((rows, V), device=DEV).scatter_add_(1, h, there.float()) > 0
    count = torch.zeros((rows, V), device=DEV).scatter_add_(1, h, said)
    rep = c["rep"][:, None]
    x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
    x = x - (c["freq"][:, None] * count + c["pres"][:, None] * (count > 0))
    if c["bias"] is not None:
        used = c["bias_tokens"] >= 0
        x = x.scatter_add(1, torch.where(used, c["bias_tokens"], 0).long(), torch.where(used, c["bias"], 0.0))
    if c["masks"] is not None:
        v = torch.arange(V, device=DEV)
        allowed = (c["masks"][:, v // 32] >> (v % 32)) & 1 != 0
        x = torch.where(allowed[c["mask_of"].clamp(min=0).long()] | (c["mask_of"] < 0)[:, None], x, -math.inf)
    return {"logits": x.to(c["logits"].dtype)}


def _teacher(c):
    """The teacher's probabilities of the stored tokens with their logarithms, and what is left for the tail, in 64 bits: little
    may be left of one, and the loss is a difference of logarithms that are nearly equal."""
    log_p = c["top_logp"].double()
    p = torch.exp(log_p)
    P = p.sum(1, keepdim=True)
    if c["tail"]:
        return p, log_p, (1.0 - P).clamp(min=0.0)
    return p / P, log_p - torch.log(P), torch.zeros_like(P)


def _plain_distill(c):
    """Relative to the row's largest logit, the sums of the stored tokens and of the others apart."""
    x = c["logits"].float() * c["scale"]
    p, log_p, r = _teacher(c)
    at = torch.where(c["top"] >= 0, c["top"], c["V"]).long()
    m = x.amax(1, keepdim=True)
    e = torch.nn.functional.pad(torch.exp(x - m), (0, 1))  # a column for the unused slots
    own = torch.gather(e, 1, at).double().sum(1, keepdim=True)
    others = e.scatter_(1, at, 0.0).sum(1, keepdim=True).double()
    log_s = torch.log(own + others)
    log_tail = -torch.log1p(own / others)
    log_q = (torch.gather(x, 1, at.clamp(max=c["V"] - 1)) - m).double() - log_s
    loss = torch.where(p > 0, p * (log_p - log_q), 0.0).sum(1, keepdim=True)
    loss = loss + torch.where((r > 0) & torch.isfinite(log_tail), r * (torch.log(r) - log_tail), 0.0)
    return loss[:, 0].float(), (m + log_s)[:, 0].float(), log_tail[:, 0].float()


def _plain_distill_grad(c, lse, log_tail, weight):
    x = c["logits"].float() * c["scale"]
    p, _, r = (v.float() for v in _teacher(c))
    r = torch.where(torch.isfinite(log_tail)[:, None], r, 0.0)
    total = p.sum(1, keepdim=True) + r
    at = torch.where(c["top"] >= 0, c["top"], c["V"]).long()
    share = torch.nn.functional.pad((total - r * torch.exp(-log_tail)[:, None]).expand(x.shape), (0, 1)).scatter(1, at, total.expand(at.shape))
    dx = torch.nn.functional.pad(torch.exp(x - lse[:, None]), (0, 1)) * share
    dx = dx.scatter_add_(1, at, -p)[:, :c["V"]]
    return (dx * (c["scale"] * weight)[:, None]).to(c["logits"].dtype)


def _plain_adapters(c):
    """All adapters at once, with the other requests' parts set to zero."""
    n, r = c["count"], c["rank"]
    u = (c["x"].float() @ c["a"].float().reshape(n * r, c["K"]).t()).reshape(c["M"], n, r)
    mine = (c["ids"][:, None] == torch.arange(n, device=DEV))[:, :, None] & (torch.arange(r, device=DEV) < c["ranks"][:, None])
    u = torch.where(mine, u * c["scales"][:, None], 0.0).reshape(c["M"], n * r)
    return {"y": (c["base"].float() + u @ c["b"].float().permute(0, 2, 1).reshape(n * r, c["N"])).to(c["x"].dtype)}


def run(state):
    c, kind = state, state["kind"]
    if not own:
        if kind == "rms":
            return _plain_rms(c)
        if kind == "rms_grad":
            return _plain_rms_grad(c)
        if kind == "adjust":
            return _plain_adjust(c)
        if kind == "adapters":
            return _plain_adapters(c)
        if kind == "distill_grad":
            return {"dlogits": _plain_distill_grad(c, c["lse"], c["log_tail"], c["weight"])}
        loss, lse, log_tail = _plain_distill(c)
        if kind == "distill":
            return {"loss": loss, "lse": lse, "log_tail": log_tail}
        return {"loss": loss, "dlogits": _plain_distill_grad(c, lse, log_tail, c["weight"])}
    import paper_1704_07355_amd as Q
    if kind == "rms":
        y, total, scale, rstd = Q.qadc_rms_norm(c["x"], c["w"], c["res"], EPS, torch.float8_e4m3fn if c["e4m3"] else None)
        out = {"rstd": rstd} if total is None else {"sum": total, "rstd": rstd}
        return dict(out, y=y) if scale is None else dict(out, y=y, scale=scale)
    if kind == "rms_grad":
        dx, dw = Q.qadc_rms_norm_backward(c["dy"], c["x"], c["w"], c["rstd"], c["dsum"], workspace=c["ws"])
        return {"dx": dx, "dw": dw}
    if kind == "adjust":
        return {"logits": Q.qadc_adjust_logits(c["logits"], c["history"], c["lengths"], c["prompt"], c["rep"], c["pres"], c["freq"],
                                               c["bias_tokens"], c["bias"], c["masks"], c["mask_of"])}
    if kind == "adapters":
        return {"y": Q.qadc_add_adapters(c["adapters"], c["ids"], c["x"], c["base"], workspace=c["ws"])}
    if kind == "distill":
        loss, lse, log_tail = Q.qadc_distill(c["logits"], c["top"], c["top_logp"], c["scale"], c["tail"], workspace=c["ws"])
        return {"loss": loss, "lse": lse, "log_tail": log_tail}
    if kind == "distill_grad":
        return {"dlogits": Q.qadc_distill_backward(c["logits"], c["top"], c["top_logp"], c["lse"], c["log_tail"], c["weight"],
                                                   c["scale"], c["tail"])}
    loss, dlogits = Q.qadc_distill_step(c["logits"], c["top"], c["top_logp"], c["weight"], c["scale"], c["tail"], workspace=c["ws"])
    return {"loss": loss, "dlogits": dlogits}


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without

def work(case):
    c, kind = case, case["kind"]
    e = BYTES[c["type"]]
    if kind == "rms":
        n = c["rows"] * c["d"]
        return {"bytes": n * ((3 if c["residual"] else 1) * e + (1 if c["e4m3"] else e)) + c["rows"] * (8 if c["e4m3"] else 4) + 4 * c["d"],
                "flops": 6 * n}
    if kind == "rms_grad":
        n = c["rows"] * c["d"]
        return {"bytes": (4 if c["residual"] else 3) * n * e + 4 * c["rows"] + 8 * c["d"], "flops": 10 * n}
    if kind == "adjust":
        rows, V = c["rows"], c["V"]
        masks = 4 * min(rows, 64) * -(-V // 32) + 4 * rows if c["masked"] else 0
        return {"bytes": rows * (2 * V * e + 4 * c["H"] + 8 * c["B"] + 20) + masks, "flops": rows * (V + 4 * c["H"])}
    if kind == "adapters":
        M, K, N, n = c["M"], c["K"], c["N"], c["count"]
        ranks = _ranks(c)
        used = ranks if c["segments"] and M >= n else ranks[:min(n, M - (0 if c["segments"] else _rows_without(M)))]
        return {"bytes": M * (K + 2 * N) * e + 4 * M + sum(used) * (K + N) * e, "flops": 2 * M * (K + N) * sum(used) // len(used)}
    n, small = c["rows"] * c["V"], c["rows"] * (8 * c["k"] + 12)
    return {"bytes": (1 if kind == "distill" else 2) * n * e + small, "flops": (4 if kind == "distill" else 8) * n}


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits

def exact(case, seed):
    c = prepare(case, seed)
    kind = c["kind"]
    if kind == "rms":
        h, out = c["x"].double(), {}
        if c["res"] is not None:
            out["sum"] = h + c["res"].double()
            h = out["sum"].to(c["x"].dtype).double()  # the norm is that of the stream that goes on
        rms = torch.sqrt(torch.sum(h * h, 1) / c["d"] + EPS)
        y = h / rms[:, None] * c["w"].double()
        out["rstd"] = 1 / rms
        if not c["e4m3"]:
            return dict(out, y=y)
        s = torch.max(torch.abs(y), 1).values / 448
        return dict(out, y=y / s[:, None], scale=s)
    if kind == "rms_grad":
        x, dy, w, rstd = c["x"].double(), c["dy"].double(), c["w"].double(), c["rstd"].double()[:, None]
        along = torch.sum(dy * w * x, 1, keepdim=True) / c["d"]
        dx = rstd * dy * w - rstd ** 3 * along * x
        return {"dx": dx if c["dsum"] is None else dx + c["dsum"].double(), "dw": torch.sum(dy * x * rstd, 0)}
    if kind == "adjust":
        rows, V = c["rows"], c["V"]
        out = []
        for i in range(rows):
            x = c["logits"][i].double()
            n, m = int(c["lengths"][i]), int(c["prompt"][i])
            seen = torch.bincount(c["history"][i, :n].long(), minlength=V) > 0
            count = torch.bincount(c["history"][i, m:n].long(), minlength=V).double()
            rep = c["rep"][i].double()
            x = torch.where(seen & (x > 0), x / rep, torch.where(seen, x * rep, x))
            x = x - c["freq"][i].double() * count - c["pres"][i].double() * (count > 0).double()
            if c["bias"] is not None:
                some = c["bias_tokens"][i] >= 0
                x = x.index_add(0, c["bias_tokens"][i][some].long(), c["bias"][i][some].double())
            if c["masks"] is not None and int(c["mask_of"][i]) >= 0:
                word = c["masks"][int(c["mask_of"][i])].long() & 0xFFFFFFFF
                bits = torch.stack([(word >> j) & 1 for j in range(32)], 1).reshape(-1)[:V]
                x = x.masked_fill(bits == 0, -math.inf)
            out.append(x)
        return {"logits": torch.stack(out)}
    if kind == "adapters":
        y = c["base"].double()
        for a, r in enumerate(_ranks(c)):
            rows = torch.nonzero(c["ids"] == a)[:, 0]
            if rows.numel():
                u = torch.mm(c["x"][rows].double(), c["a"][a, :r].double().t().contiguous())
                y[rows] += c["scales"][a].double() * torch.mm(u, c["b"][a, :, :r].double().t().contiguous())
        return {"y": y}
    rows, V = c["rows"], c["V"]
    parts = []
    for r in range(0, rows, 512):
        x = c["logits"][r:r + 512].double() * c["scale"]
        lp = torch.log_softmax(x, 1)
        tok, tl = c["top"][r:r + 512].long(), c["top_logp"][r:r + 512].double()
        p = torch.exp(tl)
        P = torch.sum(p, 1, keepdim=True)
        rest = torch.clamp(1 - P, min=0.0) if c["tail"] else torch.zeros_like(P)
        if not c["tail"]:
            tl, p = tl - torch.log(P), p / P
        off = tok < 0
        tok = tok.masked_fill(off, 0)
        inside = torch.zeros_like(x).scatter_add_(1, tok, (~off).double()) > 0
        out_lp = torch.logsumexp(lp.masked_fill(inside, -math.inf), 1, keepdim=True)
        loss = torch.sum(torch.where(off, 0.0, p * (tl.masked_fill(off, 0.0) - torch.gather(lp, 1, tok))), 1)
        loss = loss + torch.where(rest > 0, rest * (torch.log(rest) - out_lp), 0.0)[:, 0]
        if kind == "distill":
            parts.append({"loss": loss, "lse": torch.logsumexp(x, 1), "log_tail": out_lp[:, 0]})
            continue
        if kind == "distill_grad":  # of the statistics that it is given
            lp, out_lp = x - c["lse"][r:r + 512, None].double(), c["log_tail"][r:r + 512, None].double()
        q = torch.exp(lp)
        want = torch.zeros_like(x).scatter_add_(1, tok, p.masked_fill(off, 0.0)) + torch.where(inside, 0.0, rest * q / torch.exp(out_lp))
        d = (torch.sum(p, 1, keepdim=True) + rest) * q - want
        part = {"loss": loss} if kind == "distill_step" else {}
        parts.append(dict(part, dlogits=d * c["scale"] * c["weight"][r:r + 512, None].double()))
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
