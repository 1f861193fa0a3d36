"""What is timed of the end loss and of the products with quantised weights, through the public calls of ``api.py``.

Four kinds of work, each a function below:

* ``score``        log probabilities of given tokens, entropies and top alternatives (gq_token_logprobs): perplexity of a
                   calibration sequence, or the alternatives an answer is compared by.
* ``score grad``   the end loss' gradient in the logits (gq_token_logprobs_grad), where the backward pass of the saliency step starts.
* ``linear``       activation(X W_hat^T + bias) + residual with the weights as the quantiser leaves them: 4-bit codes and a
                   table of levels per channel (gq_linear); single tokens and prompts.
* ``linear grad``  its backward pass (gq_linear_grad): the gradient of the pre-activation, in the activations' type because that is what
                   the saliency step and the layer below read, and from it those of the input (same type), levels and bias (fp32).

Codes are laid out two per byte, the lower four bits first, rows padded to whole 16 bytes; tables hold 16 levels per channel in the
activations' type, zero from m on (what gq_linear_pack writes).  Activations and gradients are drawn like those of
``synth.py``: feature scales with outliers, per-token log-normal gradient scales.  Levels are spread as a fitted codebook's
are, the middle ones used more often than the outer ones.
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
ACTIVATIONS = ("none", "relu", "silu", "gelu")
LARGEST_FLOPS = 7.4e11                # of a drawn product: what the largest listed one costs
LARGEST_LOGITS = 4096 * 32000         # of a drawn score: logits of the largest listed one


def listed():
    return [
        # One decoding step's answer with five alternatives: the smallest call.
        {"name": "score one token", "kind": "score", "n": 1, "vocab": 32000, "dtype": "bf16", "top": 5, "masked": 0.0, "ignored": 0.0},
        # A batch of answers in fp32 with twenty alternatives each over a large vocabulary.
        {"name": "score answers", "kind": "score", "n": 48, "vocab": 128000, "dtype": "fp32", "top": 20, "masked": 0.01, "ignored": 0.0},
        # Perplexity of one calibration sequence (4096 tokens): no alternatives, a few tokens not counted.
        {"name": "score sequence", "kind": "score", "n": 4096, "vocab": 32000, "dtype": "bf16", "top": 0, "masked": 0.0, "ignored": 0.02},
        # The end loss' gradient for the same sequence.
        {"name": "loss gradient sequence", "kind": "score grad", "n": 4096, "vocab": 32000, "dtype": "bf16", "entropy": False, "masked": 0.0,
         "ignored": 0.02},
        # A short ragged batch with an odd vocabulary, masked logits and a gradient of the entropy as well.
        {"name": "loss gradient ragged", "kind": "score grad", "n": 211, "vocab": 50001, "dtype": "fp16", "entropy": True, "masked": 0.05,
         "ignored": 0.3},
        # Single-token serving: attention projection (c1 of the benchmark's layers).
        {"name": "linear one token", "kind": "linear", "n": 1, "d_in": 4096, "d_out": 4096, "m": 16, "dtype": "bf16", "act": "none", "bias": False,
         "residual": False},
        # Four sequences decoded together through the largest down-projection (c3), added to the residual stream.
        {"name": "linear few tokens", "kind": "linear", "n": 4, "d_in": 28672, "d_out": 8192, "m": 16, "dtype": "bf16", "act": "none", "bias": False,
         "residual": True},
        # A prompt through an up-projection with its activation.
        {"name": "linear prompt", "kind": "linear", "n": 2048, "d_in": 4096, "d_out": 11008, "m": 16, "dtype": "bf16", "act": "silu", "bias": False,
         "residual": False},
        # A short prompt, no size a multiple of a tile, 3-bit codebooks, everything in the epilogue.
        {"name": "linear ragged", "kind": "linear", "n": 77, "d_in": 1032, "d_out": 3000, "m": 8, "dtype": "fp16", "act": "gelu", "bias": True,
         "residual": True},
        # The largest: two calibration sequences through the down-projection (c2) of a quantised model.
        {"name": "linear sequences", "kind": "linear", "n": 8192, "d_in": 11008, "d_out": 4096, "m": 16, "dtype": "bf16", "act": "none", "bias": True,
         "residual": True},
        # Backward pass of a calibration batch through a quantised attention projection.
        {"name": "linear gradient", "kind": "linear grad", "n": 2048, "d_in": 4096, "d_out": 4096, "m": 16, "dtype": "bf16", "act": "silu"},
        # A ragged one with 2-bit codebooks.
        {"name": "linear gradient ragged", "kind": "linear grad", "n": 203, "d_in": 1032, "d_out": 1408, "m": 4, "dtype": "fp16", "act": "gelu"},
    ]


def _count(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi, step=8):
    return _count(rng, lo // step, hi // step) * step


def draw(rng):
    kind = rng.choice(["score", "score", "score grad", "linear", "linear", "linear", "linear grad"])
    if kind in ("score", "score grad"):
        c = {"kind": kind, "n": _count(rng, 1, 4096), "vocab": _count(rng, 500, 160000), "dtype": rng.choice(sorted(DTYPES)),
             "masked": rng.choice([0.0, 0.01, 0.3]), "ignored": rng.choice([0.0, 0.1])}
        if kind == "score":
            c["top"] = rng.choice([0, 1, 5, 20, 32])
        else:
            c["entropy"] = rng.random() < 0.5
        while c["n"] * c["vocab"] > LARGEST_LOGITS:
            c["n"] = max(1, c["n"] // 2)
        return c
    c = {"kind": kind, "n": _count(rng, 1, 8192), "d_in": _size(rng, 256, 28672), "d_out": _size(rng, 256, 11008), "m": rng.choice([4, 8, 16]),
         "dtype": rng.choice(["bf16", "fp16"]), "act": rng.choice(ACTIVATIONS)}
    if kind == "linear":
        c["bias"], c["residual"] = rng.random() < 0.5, rng.random() < 0.5
    while 2.0 * c["n"] * c["d_in"] * c["d_out"] * (2 if kind == "linear grad" else 1) > LARGEST_FLOPS:
        c["n"] = max(1, c["n"] // 2)
    return c


# ---------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed * 7919 + 23)
    return gen


def _prepare_score(c, gen):
    n, vocab = c["n"], c["vocab"]
    x = torch.randn(n, vocab, generator=gen, device=DEV)
    x *= 1.0 + 2.0 * torch.rand(n, 1, generator=gen, device=DEV)
    targets = torch.randint(0, vocab, (n,), generator=gen, device=DEV)
    # the model mostly knows its tokens: some margin for them
    x.scatter_add_(1, targets[:, None], 6.0 * torch.rand(n, 1, generator=gen, device=DEV))
    if c["masked"]:
        # tokens a sampler has ruled out; never the target
        out = torch.rand(n, vocab, generator=gen, device=DEV) < c["masked"]
        out.scatter_(1, targets[:, None], False)
        x.masked_fill_(out, float("-inf"))
        del out
    if c["ignored"]:
        targets = torch.where(torch.rand(n, generator=gen, device=DEV) < c["ignored"], torch.full_like(targets, -100), targets)
    state = {"logits": x.to(DTYPES[c["dtype"]]), "targets": targets}
    del x
    if c["kind"] == "score grad":
        x = state["logits"].float()
        top = x.amax(1)
        x -= top[:, None]
        e = x.exp()
        s = e.sum(1)
        x.masked_fill_(x == float("-inf"), 0.0)
        state["stats"] = torch.stack((top, s.log()), 1).contiguous()
        state["entropy"] = s.log() - (e * x).sum(1) / s
        state["d_logp"] = -1e-3 * torch.exp(torch.randn(n, generator=gen, device=DEV))
        state["d_entropy"] = 1e-4 * torch.randn(n, generator=gen, device=DEV) if c["entropy"] else None
    return state


def _activations(n, d, gen, dtype):
    scale = torch.exp(0.5 * torch.randn(d, generator=gen, device=DEV))
    scale[torch.randperm(d, generator=gen, device=DEV)[:max(1, d // 100)]] *= 10.0
    return (torch.randn(n, d, generator=gen, device=DEV) * scale).to(dtype)


def _prepare_linear(c, gen):
    n, d_in, d_out, m, dtype = c["n"], c["d_in"], c["d_out"], c["m"], DTYPES[c["dtype"]]
    levels = torch.sort(0.02 * (1.0 + 0.1 * torch.randn(d_out, 1, generator=gen, device=DEV))
                        * (torch.linspace(-2.2, 2.2, m, device=DEV) + 0.1 * torch.randn(d_out, m, generator=gen, device=DEV)), dim=1).values
    table = torch.zeros(d_out, 16, dtype=dtype, device=DEV)
    table[:, :m] = levels.to(dtype)
    width = (d_in + 31) // 32 * 32
    q = torch.randn(d_out, width, generator=gen, device=DEV).mul_(m / 4.4).add_(m / 2.0).floor_().clamp_(0, m - 1).to(torch.uint8)
    q[:, d_in:] = 0
    codes = (q[:, 0::2] | (q[:, 1::2] << 4)).contiguous()
    del q
    state = {"X": _activations(n, d_in, gen, dtype), "codes": codes, "table": table}
    if c["kind"] == "linear":
        state["bias"] = (0.1 * torch.randn(d_out, generator=gen, device=DEV)).to(dtype) if c["bias"] else None
        state["residual"] = torch.randn(n, d_out, generator=gen, device=DEV).to(dtype) if c["residual"] else None
    else:
        scale = 1e-2 * torch.exp(torch.randn(n, 1, generator=gen, device=DEV))
        state["dY"] = (torch.randn(n, d_out, generator=gen, device=DEV) * scale).to(dtype)
        state["Z"] = (2.0 * torch.randn(n, d_out, generator=gen, device=DEV)).to(dtype) if c["act"] != "none" else None
        if own:
            from paper_2505_07004_b200 import api
            state["workspace"] = api.alloc_workspace(api.gq_linear_grad_workspace_bytes(n, d_in, d_out), DEV)
    return state


def prepare(case, seed):
    gen = _gen(seed)
    state = _prepare_score(case, gen) if case["kind"] in ("score", "score grad") else _prepare_linear(case, gen)
    state["case"] = case
    return state


# ---------------------------------------------------------------------------------------------- one pass
def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"score": _own_score, "score grad": _own_score_grad, "linear": _own_linear, "linear grad": _own_linear_grad}[kind](state)
    return {"score": _score, "score grad": _score_grad, "linear": _linear, "linear grad": _linear_grad}[kind](state)


def _own_score(st):
    from paper_2505_07004_b200 import api
    logp, entropy, stats, top_logp, top_ids = api.gq_token_logprobs(st["logits"], st["targets"], top=st["case"]["top"])
    out = [logp, entropy, stats]
    return out + [top_logp, top_ids] if st["case"]["top"] else out


def _own_score_grad(st):
    from paper_2505_07004_b200 import api
    return api.gq_token_logprobs_grad(st["logits"], st["targets"], st["stats"], st["entropy"], st["d_logp"], st["d_entropy"])


def _own_linear(st):
    from paper_2505_07004_b200 import api
    c = st["case"]
    return api.gq_linear(st["X"], st["codes"], st["table"], c["m"], bias=st["bias"], activation=ACTIVATIONS.index(c["act"]),
                         residual=st["residual"])


def _own_linear_grad(st):
    from paper_2505_07004_b200 import api
    c = st["case"]
    dZ, dX, d_table, d_bias = api.gq_linear_grad(st["dY"], st["X"], st["codes"], st["table"], c["m"], st["workspace"], Z=st["Z"],
                                                 activation=ACTIVATIONS.index(c["act"]))
    return [dZ, dX, d_table, d_bias]


# ---- plain forms, 32 bits
def _score(st):
    x, t, k = st["logits"].float(), st["targets"], st["case"]["top"]
    vocab = x.shape[1]
    top = x.amax(1)
    shifted = x - top[:, None]
    e = shifted.exp()
    s = e.sum(1)
    log_s = s.log()
    entropy = log_s - (e * torch.where(e == 0, torch.zeros_like(e), shifted)).sum(1) / s
    counted = (t >= 0) & (t < vocab)
    at = shifted.gather(1, torch.where(counted, t, torch.zeros_like(t))[:, None])[:, 0]
    logp = torch.where(counted, at - log_s, torch.zeros_like(at))
    out = [logp, entropy, torch.stack((top, log_s), 1)]
    if k:
        ids, values = [], []
        index = torch.arange(vocab, device=x.device, dtype=torch.int32)[None, :]
        left = torch.ones_like(x, dtype=torch.bool)
        for _ in range(k):
            best = torch.where(left, x, torch.full_like(x, float("-inf"))).amax(1, keepdim=True)
            first = torch.where(left & (x == best), index, torch.full_like(index, vocab)).amin(1, keepdim=True)
            left.scatter_(1, first.long(), False)
            ids.append(first)
            values.append(best - top[:, None] - log_s[:, None])
        out += [torch.cat(values, 1), torch.cat(ids, 1)]
    return out


def _score_grad(st):
    x, t = st["logits"].float(), st["targets"]
    vocab = x.shape[1]
    logp = x - st["stats"][:, 0:1] - st["stats"][:, 1:2]
    p = logp.exp()
    counted = (t >= 0) & (t < vocab)
    w = torch.where(counted, st["d_logp"], torch.zeros_like(st["d_logp"]))
    dx = -w[:, None] * p
    dx.scatter_add_(1, torch.where(counted, t, torch.zeros_like(t))[:, None], w[:, None])
    if st["d_entropy"] is not None:
        dx -= st["d_entropy"][:, None] * p * torch.where(p == 0, torch.zeros_like(p), logp + st["entropy"][:, None])
    return dx.to(st["logits"].dtype)


def _weights(codes, table, d_in, dtype):
    q = torch.stack((codes & 15, codes >> 4), 2).reshape(codes.shape[0], -1)[:, :d_in]
    return table.to(dtype).gather(1, q.long())


def _activate(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        sig = 1.0 / (1.0 + torch.exp(-z))
        return sig * (1.0 + z * (1.0 - sig))
    return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (0.5 / math.pi) ** 0.5


def _linear(st):
    c, x = st["case"], st["X"]
    z = x.float() @ _weights(st["codes"], st["table"], c["d_in"], torch.float32).t()
    if st["bias"] is not None:
        z = z + st["bias"].float()
    y = _activate(z, c["act"])
    if st["residual"] is not None:
        y = y + st["residual"].float()
    return y.to(x.dtype)


def _linear_grad(st):
    c, x = st["case"], st["X"]
    dz = st["dY"].float()
    if c["act"] != "none":
        dz = dz * _slope(st["Z"].float(), c["act"])
    out = dz.to(x.dtype)
    dz = out.float()
    dx = dz @ _weights(st["codes"], st["table"], c["d_in"], torch.float32)
    dw = dz.t() @ x.float()
    q = torch.stack((st["codes"] & 15, st["codes"] >> 4), 2).reshape(c["d_out"], -1)[:, :c["d_in"]]
    d_table = torch.stack([torch.where(q == level, dw, torch.zeros_like(dw)).sum(1) for level in range(c["m"])], 1)
    return [out, dx.to(x.dtype), d_table, dz.sum(0)]


# ---------------------------------------------------------------------------------------------- work
def work(case):
    c = case
    if c["kind"] == "score":
        cells = c["n"] * c["vocab"]
        return {"bytes": cells * BYTES[c["dtype"]] + c["n"] * (8 + 16 + 8 * c["top"]), "flops": 5.0 * cells}
    if c["kind"] == "score grad":
        cells = c["n"] * c["vocab"]
        return {"bytes": 2 * cells * BYTES[c["dtype"]] + c["n"] * (8 + 16 + (4 if c["entropy"] else 0)),
                "flops": (8.0 if c["entropy"] else 4.0) * cells}
    n, d_in, d_out = c["n"], c["d_in"], c["d_out"]
    weights = d_out * ((d_in + 31) // 32 * 16) + d_out * 32
    if c["kind"] == "linear":
        moved = 2 * n * d_in + 2 * n * d_out * (2 if c["residual"] else 1) + (2 * d_out if c["bias"] else 0)
        return {"bytes": moved + weights, "flops": 2.0 * n * d_in * d_out}
    moved = 2 * n * d_in * 2 + 2 * n * d_out * (3 if c["act"] != "none" else 2) + 4 * d_out * (c["m"] + 1)
    return {"bytes": moved + weights, "flops": 4.0 * n * d_in * d_out}


# ---------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind in ("score", "score grad"):
        rows = [_exact_rows(st, case, lo, min(case["n"], lo + 256)) for lo in range(0, case["n"], 256)]
        if kind == "score grad":
            return torch.cat(rows)
        return [torch.cat([r[i] for r in rows]) for i in range(len(rows[0]))]
    x = st["X"].double()
    q = torch.empty(case["d_out"], st["codes"].shape[1] * 2, dtype=torch.int64, device=DEV)
    q[:, 0::2] = st["codes"] % 16
    q[:, 1::2] = st["codes"] // 16
    q = q[:, :case["d_in"]]
    level = st["table"].double()
    w = torch.zeros(case["d_out"], case["d_in"], dtype=torch.float64, device=DEV)
    for l in range(case["m"]):
        w += (q == l) * level[:, l:l + 1]
    if kind == "linear":
        z = torch.einsum("ic,jc->ij", x, w)
        if st["bias"] is not None:
            z += st["bias"].double()
        if case["act"] == "relu":
            z = z.clamp_min(0.0)
        elif case["act"] == "silu":
            z = z * torch.sigmoid(z)
        elif case["act"] == "gelu":
            z = z * torch.special.ndtr(z)
        if st["residual"] is not None:
            z += st["residual"].double()
        return z
    dz = st["dY"].double()
    if case["act"] != "none":
        z = st["Z"].double()
        if case["act"] == "relu":
            dz = torch.where(z > 0, dz, 0.0)
        elif case["act"] == "silu":
            dz = dz * (torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z))
        else:
            dz = dz * (torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
    kept = dz
    dz = dz.to(st["dY"].dtype).double()                  # what the other gradients are defined by
    dx = torch.einsum("ij,jc->ic", dz, w)
    dw = torch.einsum("ij,ic->jc", dz, x)
    d_table = torch.zeros(case["d_out"], case["m"], dtype=torch.float64, device=DEV)
    d_table.scatter_add_(1, q, dw)
    return [kept, dx, d_table, torch.einsum("ij->j", dz)]


def _exact_rows(st, case, lo, hi):
    x, t = st["logits"][lo:hi].double(), st["targets"][lo:hi]
    counted = (t >= 0) & (t < case["vocab"])
    hit = torch.where(counted, t, 0)[:, None]
    if case["kind"] == "score":
        lse = torch.logsumexp(x, 1, keepdim=True)
        logp = x - lse
        entropy = -torch.special.xlogy(logp.exp(), logp.exp()).sum(1)
        top = x.max(1).values
        out = [torch.where(counted, logp.gather(1, hit)[:, 0], 0.0), entropy, torch.stack((top, lse[:, 0] - top), 1)]
        if case["top"]:
            ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["top"]]
            out += [logp.gather(1, ids), ids.int()]
        return out
    stats, w = st["stats"][lo:hi].double(), torch.where(counted, st["d_logp"][lo:hi].double(), 0.0)[:, None]
    logp = x - stats.sum(1, keepdim=True)
    p = logp.exp()
    dx = -w * p
    dx.scatter_add_(1, hit, w)
    if st["d_entropy"] is not None:
        dx -= st["d_entropy"][lo:hi].double()[:, None] * (torch.special.xlogy(p, p) + p * st["entropy"][lo:hi].double()[:, None])
    return dx
