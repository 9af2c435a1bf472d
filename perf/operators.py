"""The vocabulary ends of a language policy: what is measured of them, with their plain forms.

Three operators, each forward and backward:

  embed   rows of an embedding table for given tokens, times a scale; its gradient is the sum of the output
          gradient's rows of each token (fp32, the whole table)
  logp    log-probabilities of given tokens from logits under a temperature, with the entropy, the
          log-sum-exp and the top alternatives of each row; its gradient with respect to the logits
  head    the same log-probabilities straight from the last hidden states and the head's weight, whose
          logits are never stored; its gradients with respect to both

A token below zero marks a padded row: it has no values (zeros; top ids -1) and no gradient.
"""
import torch

own = False                                  # True: the framework's calls; False: the plain forms

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one decoding step of 64 sequences: the embedding of each one's newest token
        {"name": "embed_step", "op": "embed", "n": 64, "vocab": 32000, "d": 2048, "type": "bf16", "scale": 1.0, "pad": 0.0},
        # the prompt and action tokens of 384 chunks of 312 positions at width 1024
        {"name": "embed_batch", "op": "embed", "n": 119808, "vocab": 32000, "d": 1024, "type": "bf16", "scale": 32.0, "pad": 0.02},
        # the gradient of one short ragged batch over a small odd vocabulary, in fp32
        {"name": "embed_grad_small", "op": "embed_bwd", "n": 997, "vocab": 1003, "d": 520, "type": "f32", "scale": 1.0, "pad": 0.1},
        # the gradient of the whole training batch
        {"name": "embed_grad_batch", "op": "embed_bwd", "n": 119808, "vocab": 32000, "d": 1024, "type": "bf16", "scale": 32.0, "pad": 0.02},
        # one decoding step: the sampled tokens' log-probabilities with eight alternatives over a large odd vocabulary
        {"name": "logp_step_top8", "op": "logp", "m": 8, "vocab": 130011, "type": "bf16", "temperature": 0.7, "top": 8, "mask": True, "pad": 0.0, "gap": 0},
        # the behaviour policy's log-probabilities of 384 x 56 action tokens, with four alternatives each
        {"name": "logp_batch_top4", "op": "logp", "m": 21504, "vocab": 32000, "type": "bf16", "temperature": 1.0, "top": 4, "mask": False, "pad": 0.02, "gap": 0},
        # the gradient of a small update in fp32, rows of odd length apart by more than their length
        {"name": "logp_grad_odd", "op": "logp_bwd", "m": 1111, "vocab": 4099, "type": "f32", "temperature": 1.3, "mask": True, "pad": 0.1, "gap": 6},
        # the gradient of a training batch
        {"name": "logp_grad_batch", "op": "logp_bwd", "m": 10752, "vocab": 32000, "type": "bf16", "temperature": 1.0, "mask": False, "pad": 0.02, "gap": 0},
        # one decoding step of 16 sequences: log-probabilities straight from the hidden states
        {"name": "head_step", "op": "head", "m": 16, "d": 2048, "vocab": 32000, "temperature": 1.0, "pad": 0.0},
        # scoring a training batch under the behaviour or reference policy
        {"name": "head_batch", "op": "head", "m": 21504, "d": 1024, "vocab": 32000, "temperature": 1.0, "pad": 0.02},
        # the gradient of a ragged small batch over an odd vocabulary
        {"name": "head_grad_ragged", "op": "head_bwd", "m": 701, "d": 1024, "vocab": 5003, "temperature": 0.8, "pad": 0.1},
        # the gradient of a training batch
        {"name": "head_grad_batch", "op": "head_bwd", "m": 21504, "d": 1024, "vocab": 32000, "temperature": 1.0, "pad": 0.02},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["embed", "embed_bwd", "logp", "logp_bwd", "head", "head_bwd"])
    kind = rng.choice(["bf16", "bf16", "f32"])
    pad = rng.choice([0.0, 0.02, 0.3])
    if op in ("embed", "embed_bwd"):
        d = _spread(rng, 48, 4096)
        d = d if rng.random() < 0.25 else -(-d // 8) * 8
        size = 4 if kind == "f32" else 2
        vocab = _spread(rng, 200, min(131072, 32000 * 1024 // d))
        n = _spread(rng, 1, min(262144, 119808 * 1024 * 2 // (d * size)))
        return {"op": op, "n": n, "vocab": vocab, "d": d, "type": kind, "scale": rng.choice([1.0, 0.5, float(d) ** 0.5]), "pad": pad}
    temperature = rng.choice([1.0, 0.7, 1.6])
    if op in ("logp", "logp_bwd"):
        most = 10752 * 32000 * 2 // (4 if kind == "f32" else 2)
        vocab = _spread(rng, 200, 200000)
        m = _spread(rng, 1, min(32768, most // vocab))
        case = {"op": op, "m": m, "vocab": vocab, "type": kind, "temperature": temperature, "mask": rng.random() < 0.5, "pad": pad,
                "gap": rng.choice([0, 0, 1, 24])}
        if op == "logp":
            case["top"] = rng.choice([0, 1, 5, 16])
        return case
    d = _spread(rng, 8, 512) * 8
    vocab = _spread(rng, 200, 131072)
    m = _spread(rng, 1, min(32768, 21504 * 32000 * 1024 // (vocab * d)))
    return {"op": op, "m": m, "d": d, "vocab": vocab, "temperature": temperature, "pad": pad}


def _tokens(g, n, vocab, pad):
    """Token frequencies fall off as one over their rank, the ranks spread over the vocabulary; some rows are padded."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    rank = torch.exp(u * torch.log(torch.tensor(float(vocab + 1), dtype=torch.float64, device="cuda"))).long() - 1
    tok = (rank.clamp_(0, vocab - 1) * 7919 + 13) % vocab
    if pad:
        tok[torch.rand(n, generator=g, device="cuda") < pad] = -1
    return tok.to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    state = {"case": dict(case)}
    op = case["op"]
    if op in ("embed", "embed_bwd"):
        n, vocab, d, t = case["n"], case["vocab"], case["d"], _TYPES[case["type"]]
        state["tok"] = _tokens(g, n, vocab, case["pad"])
        if op == "embed":
            state["table"] = (normal(vocab, d) * 0.02).to(t)
        else:
            state["dout"] = (normal(n, d) * 1e-2).to(t)
        return state
    m, vocab = case["m"], case["vocab"]
    if op in ("logp", "logp_bwd"):
        t = _TYPES[case["type"]]
        logits = torch.empty(m, vocab + case["gap"], dtype=t, device="cuda")
        step = max(1, (1 << 28) // (vocab + case["gap"]))
        for lo in range(0, m, step):         # rows of a trained head: a broad floor, a few tokens well above it
            z = torch.randn(min(step, m - lo), vocab + case["gap"], generator=g, device="cuda") * 2.0
            logits[lo:lo + step] = torch.where(z > 6.0, z * 1.5, z).to(t)
        state["logits"] = logits[:, :vocab]
        state["tok"] = _tokens(g, m, vocab, case["pad"])
        if case["mask"]:                     # a grammar leaves a part of the vocabulary, in one row nothing
            cut = vocab - vocab // 3
            state["logits"][::2, cut:] = float("-inf")
            state["logits"][m // 2, :] = float("-inf")
    else:
        d = case["d"]
        state["x"] = normal(m, d).to(torch.bfloat16)
        state["w"] = (normal(vocab, d) * (1.5 / d ** 0.5)).to(torch.bfloat16)
        state["tok"] = _tokens(g, m, vocab, case["pad"])
    if op in ("logp_bwd", "head_bwd"):       # what the forward pass kept, and the loss's gradient
        if op == "logp_bwd":
            logits, scale = state["logits"], 1.0 / case["temperature"]
            rows = [_statistics(logits[lo:lo + 2048].double() * scale) for lo in range(0, m, 2048)]
        else:
            rows = [_statistics((state["x"][lo:lo + 2048].float() @ state["w"].float().t()) / case["temperature"]) for lo in range(0, m, 2048)]
        keep = state["tok"] >= 0
        state["lse"] = torch.where(keep, torch.cat([r[0] for r in rows]), 0.0).float()
        state["entropy"] = torch.where(keep, torch.cat([r[1] for r in rows]), 0.0).float()
        state["dlogp"] = normal(m) / m
        state["dent"] = torch.full((m,), -1e-3 / m, device="cuda")
    return state


def _statistics(z):
    """Log-sum-exp and entropy of each row; a row without a finite value has -inf and 0."""
    top = z.max(-1, keepdim=True).values
    top = torch.where(top == float("-inf"), torch.zeros_like(top), top)
    e = torch.exp(z - top)
    s = e.sum(-1, keepdim=True)
    lse = (top + torch.log(s)).squeeze(-1)
    zc = torch.where(e > 0, z - top, torch.zeros_like(z))
    entropy = torch.where(s > 0, torch.log(s) - (e * zc).sum(-1, keepdim=True) / s, torch.zeros_like(s)).squeeze(-1)
    return lse, entropy


def _largest(logits, k):
    """The k largest of each row and where they are, the lowest index first among equal ones."""
    bits = (logits + 0.0).float().view(torch.int32).long()
    key = torch.where(bits < 0, -(bits & 0x7FFFFFFF) - 1, bits) * (1 << 31) - torch.arange(logits.shape[1], device=logits.device)
    at = torch.topk(key, k, dim=-1).indices
    return at, torch.gather(logits, 1, at)


def _scores(z, logits, tok, scale, k):
    """Outputs of logp from the scaled logits z."""
    keep = tok >= 0
    lse, entropy = _statistics(z)
    logp = torch.gather(z, 1, tok.clamp(min=0).long()[:, None])[:, 0] - lse
    empty = lse == float("-inf")
    logp = torch.where(empty, lse, logp)
    zero = torch.zeros_like(lse)
    out = {"logp": torch.where(keep, logp, zero), "entropy": torch.where(keep, entropy, zero), "lse": torch.where(keep, lse, zero)}
    if k:
        at, top = _largest(logits, k)
        top = torch.where(empty[:, None], lse[:, None], top.to(z.dtype) * scale - lse[:, None])
        out["top_id"] = torch.where(keep[:, None], at, -1).to(torch.int32)
        out["top_logp"] = torch.where(keep[:, None], top, zero[:, None])
    return out


def _slope(z, lse, entropy, tok, dlogp, dent, scale):
    """d loss / d logits from the scaled logits z."""
    p = torch.exp(z - lse[:, None])
    live = (tok >= 0) & (lse != float("-inf"))
    p = torch.where(live[:, None], p, torch.zeros_like(p))
    g = torch.where(p > 0, -p * (dlogp[:, None] + dent[:, None] * (z - lse[:, None] + entropy[:, None])), torch.zeros_like(p))
    rows = torch.nonzero(live)[:, 0]
    g[rows, tok[rows].long()] += dlogp[rows]
    return g * scale


def _plain(state):
    case = state["case"]
    op, tok = case["op"], state["tok"]
    keep = tok >= 0
    if op == "embed":
        rows = state["table"][tok.clamp(min=0).long()].float() * case["scale"]
        return {"out": torch.where(keep[:, None], rows, 0.0).to(state["table"].dtype)}
    if op == "embed_bwd":
        grad = torch.zeros(case["vocab"], case["d"], device="cuda")
        rows = torch.where(keep[:, None], state["dout"].float() * case["scale"], 0.0)
        return {"grad": grad.index_add_(0, tok.clamp(min=0).long(), rows)}
    scale = 1.0 / case["temperature"]
    if op == "logp":
        return _scores(state["logits"].float() * scale, state["logits"], tok, scale, case["top"])
    if op == "logp_bwd":
        g = _slope(state["logits"].float() * scale, state["lse"], state["entropy"], tok, state["dlogp"], state["dent"], scale)
        return {"dlogits": g.to(state["logits"].dtype)}
    x, w = state["x"].float(), state["w"].float()
    z = (x @ w.t()) * scale
    if op == "head":
        return _scores(z, z, tok, scale, 0)
    g = _slope(z, state["lse"], state["entropy"], tok, state["dlogp"], state["dent"], scale)
    return {"dx": (g @ w).to(torch.bfloat16), "dw": g.t() @ x}


def _own(state):
    from paper_2605_16154_b200 import binding as lib
    case = state["case"]
    op, tok = case["op"], state["tok"]
    if op == "embed":
        return {"out": lib.grpo_embed(state["table"], tok, scale=case["scale"])}
    if op == "embed_bwd":
        return {"grad": lib.grpo_embed_bwd(state["dout"], tok, case["vocab"], scale=case["scale"])}
    if op == "logp":
        logp, entropy, lse, top_id, top_logp = lib.grpo_token_logp(state["logits"], tok, temperature=case["temperature"], top=case["top"])
        out = {"logp": logp, "entropy": entropy, "lse": lse}
        return {**out, "top_id": top_id, "top_logp": top_logp} if case["top"] else out
    if op == "logp_bwd":
        return {"dlogits": lib.grpo_token_logp_bwd(state["logits"], tok, state["lse"], state["entropy"], state["dlogp"], state["dent"],
                                                   temperature=case["temperature"])}
    if op == "head":
        logp, entropy, lse = lib.grpo_head_logp(state["x"], state["w"], tok, temperature=case["temperature"])
        return {"logp": logp, "entropy": entropy, "lse": lse}
    dx, dw = lib.grpo_head_logp_bwd(state["x"], state["w"], tok, state["lse"], state["entropy"], state["dlogp"], state["dent"],
                                    temperature=case["temperature"])
    return {"dx": dx, "dw": dw}


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    """Each input read once, each output written once; the products of the head as matrix products."""
    op = case["op"]
    if op in ("embed", "embed_bwd"):
        n, vocab, d = case["n"], case["vocab"], case["d"]
        size = 4 if case["type"] == "f32" else 2
        if op == "embed":
            return {"bytes": (n + min(n, vocab)) * d * size + 4 * n, "flops": n * d}
        return {"bytes": n * d * size + 4 * n + 4 * vocab * d, "flops": 2 * n * d}
    m, vocab = case["m"], case["vocab"]
    if op in ("logp", "logp_bwd"):
        size = 4 if case["type"] == "f32" else 2
        if op == "logp":
            return {"bytes": m * vocab * size + 4 * m * (4 + 2 * case["top"]), "flops": 5 * m * vocab}
        return {"bytes": 2 * m * vocab * size + 20 * m, "flops": 7 * m * vocab}
    d = case["d"]
    if op == "head":
        return {"bytes": 2 * d * (m + vocab) + 16 * m, "flops": 2 * m * vocab * d}
    return {"bytes": 2 * d * (m + vocab) + 20 * m + 2 * m * d + 4 * vocab * d, "flops": 6 * m * vocab * d}


def exact(case, seed):
    """The operators' definitions in 64 bits, a few rows at a time."""
    state = prepare(case, seed)
    op, tok = case["op"], state["tok"].long()
    f64 = torch.float64
    if op == "embed":
        out = torch.zeros(case["n"], case["d"], dtype=f64, device="cuda")
        at = torch.nonzero(tok >= 0)[:, 0]
        out[at] = state["table"].to(f64)[tok[at]] * case["scale"]
        return {"out": out}
    if op == "embed_bwd":
        grad = torch.zeros(case["vocab"], case["d"], dtype=f64, device="cuda")
        at = torch.nonzero(tok >= 0)[:, 0]
        for part in at.split(16384):
            grad.index_add_(0, tok[part], state["dout"][part].to(f64) * case["scale"])
        return {"grad": grad}
    m, vocab, heat = case["m"], case["vocab"], case["temperature"]
    rows = max(1, (1 << 26) // vocab)
    w = state["w"].to(f64) if "w" in state else None
    parts, dw = [], None
    for lo in range(0, m, rows):
        hi = min(m, lo + rows)
        t = tok[lo:hi]
        raw = state["x"][lo:hi].to(f64) @ w.t() if w is not None else state["logits"][lo:hi].to(f64)
        z = raw / heat
        live = (t >= 0) & torch.isfinite(z).any(-1)
        z = torch.where(live[:, None], z, torch.zeros_like(z))
        full = torch.logsumexp(z, -1)
        lp = z - full[:, None]
        p = lp.exp()
        plp = torch.where(p > 0, p * lp, torch.zeros_like(p))
        at = t.clamp(min=0)[:, None]
        if op in ("logp", "head"):
            none = torch.where(t >= 0, float("-inf"), 0.0).to(f64)
            one = {"logp": torch.where(live, lp.gather(1, at)[:, 0], none), "entropy": torch.where(live, -plp.sum(-1), 0.0),
                   "lse": torch.where(live, full, none)}
            if case.get("top"):
                order = torch.sort(raw, dim=-1, descending=True, stable=True)
                best = order.indices[:, :case["top"]]
                one["top_id"] = torch.where((t >= 0)[:, None], best, -1).to(torch.int32)
                one["top_logp"] = torch.where(live[:, None], lp.gather(1, best), none[:, None])
            parts.append(one)
            continue
        a, b = state["dlogp"][lo:hi].to(f64)[:, None], state["dent"][lo:hi].to(f64)[:, None]
        ent = -plp.sum(-1, keepdim=True)
        g = -a * p - b * (plp + p * ent)
        g.scatter_add_(1, at, a)
        g = torch.where(live[:, None], g, torch.zeros_like(g)) / heat
        if op == "logp_bwd":
            parts.append({"dlogits": g if m * vocab <= (1 << 29) else g.float()})
        else:
            parts.append({"dx": g @ w})
            step = g.t() @ state["x"][lo:hi].to(f64)
            dw = step if dw is None else dw.add_(step)
    out = {k: torch.cat([q[k] for q in parts]) for k in parts[0]}
    if dw is not None:
        out["dw"] = dw
    return out
