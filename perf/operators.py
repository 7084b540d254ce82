"""Cases of the inner training step's operators: gradient clipping, the embedding,
token log probabilities and the gated feed-forward block.

A worker of the outer step trains between two of them; these are the operators of
its step around the library's matrix products.  ``run`` computes a case in its
plain form (elementary torch operations in 32 bits, rounded once at the end) or,
where ``own`` is true, with the package's kernels.  ``exact`` has the same outputs
from the definitions in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


# --------------------------------------------------------------------------
# Cases
# --------------------------------------------------------------------------

def listed():
    return [
        # the gradients of one decoder block (9 tensors), clipped into a second buffer
        {"name": "clip block f32", "op": "clip", "blocks": 1, "dim": 768, "hidden": 2048, "vocab": 0, "dtype": "f32",
         "max_norm": 1.0},
        # 888M parameters: bfloat16 matrices and float32 gains, 145 tensors, clipped
        {"name": "clip 16L bf16", "op": "clip", "blocks": 16, "dim": 2048, "hidden": 5632, "vocab": 32000,
         "dtype": "bf16", "max_norm": 1.0},
        # the next tokens of 64 sequences that are being generated
        {"name": "embed 64", "op": "embed", "tokens": 64, "dim": 2048, "vocab": 32000, "dtype": "bf16", "scale": 1.0},
        # a ragged batch of a model of odd width, float32 throughout
        {"name": "embed grad 5001 d612", "op": "embed_grad", "tokens": 5001, "dim": 612, "vocab": 32000,
         "dtype": "f32", "scale": 24.7},
        # 16 sequences of 2048 tokens, bfloat16 activations into a float32 gradient
        {"name": "embed grad 32768 d2048", "op": "embed_grad", "tokens": 32768, "dim": 2048, "vocab": 32000,
         "dtype": "bf16", "scale": 1.0},
        # four sequences being generated: the sampled tokens' log probabilities and 8 alternatives
        {"name": "logprob 4 top8", "op": "logprob", "rows": 4, "vocab": 32000, "dtype": "bf16", "scale": 1.25,
         "top": 8},
        # the validation loss of two sequences with entropy and the 5 best alternatives
        {"name": "logprob 4096 top5 f32", "op": "logprob", "rows": 4096, "vocab": 32000, "dtype": "f32", "scale": 1.0,
         "top": 5},
        # the loss of a training step and its gradient, four sequences
        {"name": "logprob grad 8192", "op": "logprob_grad", "rows": 8192, "vocab": 32000, "dtype": "bf16",
         "scale": 1.0, "top": 0},
        # one token of one sequence being generated
        {"name": "ffn token", "op": "ffn", "tokens": 1, "dim": 2048, "hidden": 5632, "dtype": "bf16", "act": "silu"},
        # one sequence of 2048 tokens through the d = 768 model's block
        {"name": "ffn 2048 d768", "op": "ffn", "tokens": 2048, "dim": 768, "hidden": 2048, "dtype": "bf16",
         "act": "silu"},
        # ragged sizes, float32 throughout: gradients of the input and both weights
        {"name": "ffn grad 1000 d612 f32", "op": "ffn_grad", "tokens": 1000, "dim": 612, "hidden": 1637,
         "dtype": "f32", "act": "gelu"},
        # eight sequences of 2048 tokens through the d = 2048 model's block, backward
        {"name": "ffn grad 16384 d2048", "op": "ffn_grad", "tokens": 16384, "dim": 2048, "hidden": 5632,
         "dtype": "bf16", "act": "silu"},
    ]


def _spread(rng, lo, hi, step=1):
    """A multiple of ``step`` of [lo, hi], uniform in its logarithm."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    n = min(hi, max(lo, n // step * step))
    return n - step if n == 3072 else n


def _width(rng, lo, hi):
    """A width: a multiple of 64 half of the time, any integer otherwise."""
    return _spread(rng, lo, hi, 64 if rng.random() < 0.5 else 1)


def draw(rng):
    op = rng.choice(("clip", "embed", "embed_grad", "logprob", "logprob_grad", "ffn", "ffn_grad"))
    dtype = rng.choice(("f32", "bf16"))
    if op == "clip":
        return {"op": op, "blocks": _spread(rng, 1, 16), "dim": _width(rng, 64, 1024), "hidden": _width(rng, 128, 2816),
                "vocab": rng.choice((0, _spread(rng, 500, 32000))), "dtype": dtype,
                "max_norm": rng.choice((1.0, 0.25, 1e6))}
    if op in ("embed", "embed_grad"):
        return {"op": op, "tokens": _spread(rng, 1, 32768), "dim": _width(rng, 64, 2048),
                "vocab": _spread(rng, 500, 32000), "dtype": dtype, "scale": rng.choice((1.0, 24.7, 0.125))}
    if op in ("logprob", "logprob_grad"):
        # the largest listed case has 2^28 logits
        vocab = _spread(rng, 500, 128000)
        rows = _spread(rng, 1, max(1, min(8192, 2 ** 27 // vocab)))
        return {"op": op, "rows": rows, "vocab": vocab, "dtype": dtype, "scale": rng.choice((1.0, 1.25, 0.7)),
                "top": rng.choice((0, 1, 5, 8, 20)) if op == "logprob" else 0}
    # float32 products take several times a bfloat16 one's work: fewer tokens there
    return {"op": op, "tokens": _spread(rng, 1, 16384 if dtype == "bf16" else 2048), "dim": _width(rng, 64, 2048),
            "hidden": _width(rng, 128, 5632), "dtype": dtype, "act": rng.choice(("silu", "gelu"))}


def _layout(case):
    """(matrix shapes, gain lengths) of a model's gradients."""
    d, f = case["dim"], case["hidden"]
    mats = [(d, d), (d, d), (d, d), (d, d), (f, d), (f, d), (d, f)] * case["blocks"]
    if case["vocab"]:
        mats.append((case["vocab"], d))
    return mats, [d] * (2 * case["blocks"])


def work(case):
    op, b = case["op"], SIZE[case["dtype"]]
    if op == "clip":
        # every gradient read once and written once (the norm has to be known before the writes)
        mats, gains = _layout(case)
        m, g = sum(r * c for r, c in mats), sum(gains)
        return {"bytes": 2 * (m * b + g * 4), "flops": 3 * (m + g)}
    if op == "embed":
        return {"bytes": case["tokens"] * (8 + 2 * case["dim"] * b), "flops": case["tokens"] * case["dim"]}
    if op == "embed_grad":
        return {"bytes": case["tokens"] * (8 + case["dim"] * b) + case["vocab"] * case["dim"] * 4,
                "flops": case["tokens"] * case["dim"]}
    if op == "logprob":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * b + case["rows"] * (20 + 12 * case["top"]), "flops": 5 * n}
    if op == "logprob_grad":
        n = case["rows"] * case["vocab"]
        return {"bytes": 2 * n * b + case["rows"] * 28, "flops": 10 * n}
    t, d, f = case["tokens"], case["dim"], case["hidden"]
    if op == "ffn":
        return {"bytes": (t * d + 2 * f * d + t * f) * b, "flops": 4 * t * d * f}
    return {"bytes": (2 * t * d + 4 * f * d + t * f) * b, "flops": 12 * t * d * f}


# --------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------

def _ids(n, vocab, g, dev, pad):
    """Token ids whose counts fall as 1 / rank, as a text's do, with a few positions
    that hold no token (-1)."""
    u = torch.rand(n, generator=g, device=dev, dtype=torch.float64)
    ids = (torch.pow(float(vocab + 1), u) - 1).to(torch.int64).clamp_(0, vocab - 1)
    if pad:
        ids[torch.rand(n, generator=g, device=dev) < pad] = -1
    return ids


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) * 7919 + 17)
    dt, op = DTYPES[case["dtype"]], case["op"]

    def randn(*shape, std=1.0, dtype=torch.float32):
        return torch.randn(*shape, generator=g, device=dev).mul_(std).to(dtype)

    if op == "clip":
        # flat buffers that hold the tensors one after the other, and the tensors in them
        mats, gains = _layout(case)
        flat_m = randn(sum(r * c for r, c in mats), std=1e-3, dtype=dt)
        flat_g = randn(sum(gains), std=1e-2)
        state = {"flat": (flat_m, flat_g), "grads": _views(flat_m, mats) + _views(flat_g, [(n,) for n in gains])}
        flat_out = (torch.empty_like(flat_m), torch.empty_like(flat_g))
        state["flat_out"] = flat_out
        state["outs"] = _views(flat_out[0], mats) + _views(flat_out[1], [(n,) for n in gains])
    elif op == "embed":
        state = {"table": randn(case["vocab"], case["dim"], std=0.02, dtype=dt),
                 "ids": _ids(case["tokens"], case["vocab"], g, dev, 0.0)}
    elif op == "embed_grad":
        state = {"ids": _ids(case["tokens"], case["vocab"], g, dev, 0.02),
                 "dout": randn(case["tokens"], case["dim"], std=1e-3, dtype=dt)}
    elif op in ("logprob", "logprob_grad"):
        rows, vocab = case["rows"], case["vocab"]
        targets = _ids(rows, vocab - vocab // 100, g, dev, 0.03 if op == "logprob_grad" else 0.0)
        logits = randn(rows, vocab, std=2.0)
        # a model that has learnt something: the target stands out; the vocabulary's padding is masked
        logits[torch.arange(rows, device=dev), targets.clamp(min=0)] += 6.0
        logits[:, vocab - vocab // 100:] = -math.inf
        state = {"logits": logits.to(dt), "targets": targets}
        if op == "logprob_grad":
            state["dlogprob"] = torch.where(targets >= 0, -1.0 / rows, 0.0).to(torch.float32)
            state["dentropy"] = torch.full((rows,), -0.01 / rows, device=dev)
    else:
        t, d, f = case["tokens"], case["dim"], case["hidden"]
        state = {"x": randn(t, d, dtype=dt), "w_gate": randn(f, d, std=0.02, dtype=dt),
                 "w_up": randn(f, d, std=0.02, dtype=dt)}
        if op == "ffn_grad":
            state["dout"] = randn(t, f, std=1e-3, dtype=dt)
    state["case"] = dict(case)
    return state


def _views(flat, shapes):
    sizes = [math.prod(s) for s in shapes]
    return [p.view(s) for p, s in zip(flat.split(sizes), shapes)] if sizes else []


# --------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    return (_RUN_OWN if own else _RUN_PLAIN)[op](state, state["case"])


def _own_clip(s, c):
    import paper_2607_03011_amd as iso
    norm = iso.clip_grads(s["grads"], c["max_norm"], out=s["outs"])
    return {"norm": norm, "matrices": s["flat_out"][0], "gains": s["flat_out"][1]}


def _own_embed(s, c):
    import paper_2607_03011_amd as iso
    return iso.embedding(s["table"], s["ids"], scale=c["scale"])


def _own_embed_grad(s, c):
    import paper_2607_03011_amd as iso
    return iso.embedding_backward(s["ids"], s["dout"], c["vocab"], scale=c["scale"], out_dtype=torch.float32)


def _own_logprob(s, c):
    import paper_2607_03011_amd as iso
    r = iso.token_logprobs(s["logits"], s["targets"], scale=c["scale"], top_k=c["top"])
    out = {"logprob": r.logprob, "entropy": r.entropy, "lse": r.lse}
    return dict(out, top_logprob=r.top_logprob, top_index=r.top_index) if c["top"] else out


def _own_logprob_grad(s, c):
    import paper_2607_03011_amd as iso
    r = iso.token_logprobs(s["logits"], s["targets"], scale=c["scale"])
    d = iso.token_logprobs_backward(s["logits"], s["targets"], r.lse, s["dlogprob"], entropy=r.entropy,
                                    dentropy=s["dentropy"], scale=c["scale"])
    return {"logprob": r.logprob, "entropy": r.entropy, "dlogits": d}


def _own_ffn(s, c):
    import paper_2607_03011_amd as iso
    return iso.gated_ffn(s["x"], s["w_gate"], s["w_up"], act=c["act"])


def _own_ffn_grad(s, c):
    import paper_2607_03011_amd as iso
    dx, dwg, dwu = iso.gated_ffn_backward(s["x"], s["w_gate"], s["w_up"], s["dout"], act=c["act"])
    return {"dx": dx, "dw_gate": dwg, "dw_up": dwu}


def _plain_clip(s, c):
    norm = torch.stack([t.float().square().sum() for t in s["grads"]]).sum().sqrt()
    coef = torch.where(norm > c["max_norm"], c["max_norm"] / norm, torch.ones_like(norm))
    m, g = s["flat"]
    return {"norm": torch.stack([norm, coef]), "matrices": (m.float() * coef).to(m.dtype), "gains": g * coef}


def _plain_embed(s, c):
    return (s["table"][s["ids"]].float() * c["scale"]).to(s["table"].dtype)


def _plain_embed_grad(s, c):
    d = torch.zeros(c["vocab"] + 1, c["dim"], device=s["ids"].device)
    at = torch.where(s["ids"] >= 0, s["ids"], c["vocab"])
    d.index_add_(0, at, s["dout"].float())
    return d[:-1] * c["scale"]


def _softmax_parts(s, c):
    z = s["logits"].float() * c["scale"]
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    lse = m + torch.log(total)
    p = e / total
    logp = z - lse
    entropy = -torch.where(p > 0, p * logp, 0.0).sum(1)
    t = s["targets"]
    logprob = torch.where(t >= 0, logp.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0)
    return z, p, logp, lse[:, 0], entropy, logprob


def _plain_logprob(s, c):
    z, p, logp, lse, entropy, logprob = _softmax_parts(s, c)
    out = {"logprob": logprob, "entropy": entropy, "lse": lse}
    if not c["top"]:
        return out
    # the order of the values as integers, ties by the lower index
    bits = (s["logits"].float() + 0.0).view(torch.int32).to(torch.int64)
    bits = torch.where(bits < 0, -2147483649 - bits, bits)
    key = bits * 2 ** 31 + (2 ** 31 - 1 - torch.arange(c["vocab"], device=bits.device))
    index = torch.topk(key, c["top"], dim=1).indices
    return dict(out, top_logprob=logp.gather(1, index), top_index=index)


def _plain_logprob_grad(s, c):
    z, p, logp, lse, entropy, logprob = _softmax_parts(s, c)
    dl = torch.where(s["targets"] >= 0, s["dlogprob"], 0.0)
    d = -p * dl[:, None] - s["dentropy"][:, None] * torch.where(p > 0, p * (logp + entropy[:, None]), 0.0)
    d.scatter_add_(1, s["targets"].clamp(min=0)[:, None], dl[:, None])
    return {"logprob": logprob, "entropy": entropy, "dlogits": (d * c["scale"]).to(s["logits"].dtype)}


def _gate(g, act):
    """act(g) and its derivative."""
    if act == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    cdf = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
    return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))


def _plain_ffn(s, c):
    x, wg, wu = s["x"].float(), s["w_gate"].float(), s["w_up"].float()
    return (_gate(x @ wg.T, c["act"])[0] * (x @ wu.T)).to(s["x"].dtype)


def _plain_ffn_grad(s, c):
    x, wg, wu, dout = s["x"].float(), s["w_gate"].float(), s["w_up"].float(), s["dout"].float()
    a, da = _gate(x @ wg.T, c["act"])
    dg, du = dout * (x @ wu.T) * da, dout * a
    dt = s["x"].dtype
    return {"dx": (dg @ wg + du @ wu).to(dt), "dw_gate": (dg.T @ x).to(dt), "dw_up": (du.T @ x).to(dt)}


_RUN_OWN = {"clip": _own_clip, "embed": _own_embed, "embed_grad": _own_embed_grad, "logprob": _own_logprob,
            "logprob_grad": _own_logprob_grad, "ffn": _own_ffn, "ffn_grad": _own_ffn_grad}
_RUN_PLAIN = {"clip": _plain_clip, "embed": _plain_embed, "embed_grad": _plain_embed_grad, "logprob": _plain_logprob,
              "logprob_grad": _plain_logprob_grad, "ffn": _plain_ffn, "ffn_grad": _plain_ffn_grad}


# --------------------------------------------------------------------------
# The definitions in 64 bits
# --------------------------------------------------------------------------

def exact(case, seed):
    """What run() returns for these inputs, from the definitions in 64 bits."""
    s, op = prepare(case, seed), case["op"]
    if op == "clip":
        sq = sum(float(torch.linalg.vector_norm(t, dtype=torch.float64)) ** 2 for t in s["flat"])
        norm = math.sqrt(sq)
        coef = min(1.0, case["max_norm"] / norm)
        return {"norm": torch.tensor([norm, coef], dtype=torch.float64, device="cuda"),
                "matrices": s["flat"][0].double() * coef, "gains": s["flat"][1].double() * coef}
    if op == "embed":
        return torch.index_select(s["table"], 0, s["ids"]).double().mul_(case["scale"])
    if op == "embed_grad":
        keep = s["ids"] >= 0
        d = torch.zeros(case["vocab"], case["dim"], dtype=torch.float64, device="cuda")
        d.index_put_((s["ids"][keep],), s["dout"][keep].double() * case["scale"], accumulate=True)
        return d
    if op in ("logprob", "logprob_grad"):
        return _exact_logprob(s, case)
    x, wg, wu = s["x"].double(), s["w_gate"].double(), s["w_up"].double()
    g, u = torch.mm(x, wg.t()), torch.mm(x, wu.t())
    if case["act"] == "silu":
        sg = torch.sigmoid(g)
        a = g * sg
        da = sg + a * (1 - sg)
    else:
        cdf = torch.special.ndtr(g)
        a = g * cdf
        da = cdf + g * torch.exp(-g ** 2 / 2) / math.sqrt(2 * math.pi)
    if op == "ffn":
        return a * u
    dh = s["dout"].double()
    dg, du = dh * u * da, dh * a
    return {"dx": torch.mm(dg, wg) + torch.mm(du, wu), "dw_gate": torch.mm(dg.t(), x), "dw_up": torch.mm(du.t(), x)}


def _exact_logprob(s, case):
    rows, top = case["rows"], case["top"]
    parts = []
    for r in range(0, rows, 1024):
        z = s["logits"][r:r + 1024].double() * case["scale"]
        t = s["targets"][r:r + 1024]
        lse = torch.logsumexp(z, 1)
        logp = z - lse[:, None]
        p = torch.exp(logp)
        plogp = torch.special.xlogy(p, p)
        entropy = -plogp.sum(1)
        valid = t >= 0
        picked = logp[torch.arange(len(t), device=t.device), t.clamp(min=0)]
        one = {"logprob": torch.where(valid, picked, torch.zeros_like(picked)), "entropy": entropy}
        if case["op"] == "logprob":
            one["lse"] = lse
            if top:
                value, index = torch.sort(z, dim=1, descending=True, stable=True)
                one["top_logprob"] = value[:, :top] - lse[:, None]
                one["top_index"] = index[:, :top]
        else:
            dl = s["dlogprob"][r:r + 1024].double() * valid
            de = s["dentropy"][r:r + 1024].double()
            d = torch.nn.functional.one_hot(t.clamp(min=0), case["vocab"]) * dl[:, None] - p * dl[:, None]
            d -= de[:, None] * (plogp + p * entropy[:, None])
            one["dlogits"] = d * case["scale"]
        parts.append(one)
    return {k: torch.cat([q[k] for q in parts]) for k in parts[0]}
