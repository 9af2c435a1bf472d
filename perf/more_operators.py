"""The rollout side of a policy: what is measured of it, with the plain forms.

Three operators:

  rotary  rotary positions of given rows: both layouts, a part of the head or all of it, frequencies scaled for long
          contexts; its gradient is the opposite rotation
  append  new tokens enter a paged cache: their queries and keys are rotated, keys and values go to their pages
  attend  attention of new tokens over the paged cache: causal, grouped heads, from one new token a sequence (a decoding
          step) to long chunks of them, over everything before or over a window of it and a few first tokens

Sequence s holds seq_len[s] tokens, its new ones included; token j is in slot j % page of page table[s][j // page].  The
rows of its new tokens are q_off[s] .. q_off[s + 1] - 1, and the last row is the sequence's last token.
"""
import math
import random

import torch

own = False                                  # True: the framework's calls; False: the plain forms

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # queries of one training batch: 384 chunks of 312 positions, 16 heads of 64
        {"name": "rotary_batch", "op": "rotary", "n": 119808, "heads": 16, "dim": 64, "rot": 64, "type": "bf16", "layout": "half",
         "scaling": "none", "far": 312, "inverse": False},
        # the gradient of a small update in fp32 far into a long context, half of each head in the interleaved layout
        {"name": "rotary_grad_far", "op": "rotary", "n": 3001, "heads": 12, "dim": 96, "rot": 48, "type": "f32", "layout": "interleaved",
         "scaling": "parts", "far": 1000000, "inverse": True},
        # one decoding step of 64 rollouts
        {"name": "append_step", "op": "append", "seqs": 64, "new_lo": 1, "new_hi": 1, "len_lo": 257, "len_hi": 312, "heads": 16, "kv": 16,
         "dim": 128, "rot": 128, "page": 16, "type": "bf16", "layout": "half", "scaling": "none", "heads_first": False},
        # the observation prefixes of 384 chunks
        {"name": "append_prefix", "op": "append", "seqs": 384, "new_lo": 256, "new_hi": 256, "len_lo": 256, "len_hi": 256, "heads": 16,
         "kv": 8, "dim": 64, "rot": 64, "page": 64, "type": "bf16", "layout": "half", "scaling": "linear", "heads_first": False},
        # one robot asks for its next action token
        {"name": "attend_step_one", "op": "attend", "seqs": 1, "new_lo": 1, "new_hi": 1, "len_lo": 257, "len_hi": 312, "heads": 16, "kv": 16,
         "dim": 64, "page": 16, "type": "bf16", "window": 0, "sinks": 0, "heads_first": False},
        # a decoding step of 256 rollouts that kept their earlier chunks
        {"name": "attend_step_batch", "op": "attend", "seqs": 256, "new_lo": 1, "new_hi": 1, "len_lo": 500, "len_hi": 8192, "heads": 16,
         "kv": 4, "dim": 128, "page": 32, "type": "bf16", "window": 0, "sinks": 0, "heads_first": False},
        # a decoding step of two sequences with a very long history
        {"name": "attend_step_far", "op": "attend", "seqs": 2, "new_lo": 1, "new_hi": 1, "len_lo": 100000, "len_hi": 131072, "heads": 32,
         "kv": 8, "dim": 128, "page": 16, "type": "bf16", "window": 0, "sinks": 0, "heads_first": True},
        # eight tokens of each of 40 sequences at once over a window and four first tokens
        {"name": "attend_few_window", "op": "attend", "seqs": 40, "new_lo": 5, "new_hi": 8, "len_lo": 1500, "len_hi": 9001, "heads": 12,
         "kv": 4, "dim": 64, "page": 16, "type": "bf16", "window": 1024, "sinks": 4, "heads_first": False},
        # the observation prefixes of 384 chunks
        {"name": "attend_prefix", "op": "attend", "seqs": 384, "new_lo": 256, "new_hi": 256, "len_lo": 256, "len_hi": 256, "heads": 16,
         "kv": 16, "dim": 64, "page": 64, "type": "bf16", "window": 0, "sinks": 0, "heads_first": False},
        # long chunks of new tokens behind a long history
        {"name": "attend_chunk_far", "op": "attend", "seqs": 8, "new_lo": 1024, "new_hi": 1024, "len_lo": 4096, "len_hi": 8192, "heads": 16,
         "kv": 4, "dim": 128, "page": 16, "type": "bf16", "window": 0, "sinks": 0, "heads_first": False},
        # ragged chunks over a window and a few first tokens, pages that do not divide a tile
        {"name": "attend_chunk_window", "op": "attend", "seqs": 5, "new_lo": 301, "new_hi": 997, "len_lo": 1001, "len_hi": 6007, "heads": 10,
         "kv": 2, "dim": 64, "page": 48, "type": "bf16", "window": 777, "sinks": 5, "heads_first": True},
        # a small ragged batch in fp32: some sequences decode, some bring a few tokens
        {"name": "attend_ragged_f32", "op": "attend", "seqs": 37, "new_lo": 1, "new_hi": 40, "len_lo": 3, "len_hi": 701, "heads": 6, "kv": 2,
         "dim": 64, "page": 16, "type": "f32", "window": 0, "sinks": 0, "heads_first": False},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["rotary", "append", "attend", "attend", "attend"])
    kind = rng.choice(["bf16", "bf16", "bf16", "f32"])
    layout, scaling = rng.choice(["half", "interleaved"]), rng.choice(["none", "linear", "parts"])
    size = 4 if kind == "f32" else 2
    if op == "rotary":
        dim = rng.choice([32, 64, 80, 96, 128, 256])
        heads = _spread(rng, 1, 48)
        n = _spread(rng, 1, 119808 * 1024 * 2 // (heads * dim * size))
        return {"op": op, "n": min(n, 1 << 20), "heads": heads, "dim": dim, "rot": rng.choice([dim, dim, dim // 2, dim // 4]), "type": kind,
                "layout": layout, "scaling": scaling, "far": _spread(rng, 56, 1 << 20), "inverse": rng.random() < 0.4}
    dim = rng.choice([32, 64, 64, 128, 128])
    kv = rng.choice([1, 2, 3, 4, 8, 16])
    heads = kv * rng.choice([1, 1, 2, 3, 4, 5, 8])
    case = {"op": op, "heads": heads, "kv": kv, "dim": dim, "page": rng.choice([8, 16, 16, 24, 32, 48, 64, 128, 256]), "type": kind,
            "heads_first": rng.random() < 0.3}
    step = rng.choice(["one", "one", "few", "chunk", "chunk"])
    if op == "append":
        new = 1 if step == "one" else _spread(rng, 2, 16) if step == "few" else _spread(rng, 17, 2048)
        far = new + _spread(rng, 1, 4096)
        seqs = _spread(rng, 1, max(1, min(512, (1 << 27) // (new * (heads + 2 * kv) * dim * size), (1 << 27) // (far * kv * dim * size))))
        case.update(seqs=seqs, new_lo=rng.choice([1, new]), new_hi=new, len_lo=rng.choice([new, far]), len_hi=far, rot=rng.choice([dim, dim, dim // 2]),
                    layout=layout, scaling=scaling)
        return case
    far = _spread(rng, 40, 131072)
    part = 8 if kind == "f32" else 1         # fp32 is the mode for checks: less work, the same shapes
    cells, keys = (1 << 36) // (part * max(dim, 64)), (3 << 27) // (part * kv * dim)
    new = 1 if step == "one" else _spread(rng, 2, 16) if step == "few" else _spread(rng, 17, 2048)
    new = min(new, far, max(1, cells // (heads * far)))
    seqs = _spread(rng, 1, max(1, min(512, keys // far, cells // (heads * far * new))))
    window = rng.choice([0, 0, _spread(rng, 16, 8192)])
    case.update(seqs=seqs, new_lo=rng.choice([1, new]), new_hi=new, len_lo=rng.choice([new, max(new, far // 2)]), len_hi=far, window=window,
                sinks=rng.choice([0, 1, 4, 100]) if window else 0)
    return case


def _lengths(case):
    """(new tokens, tokens in all) of each sequence: a part of the case, the same for every seed."""
    rng = random.Random(case["seqs"] * 1000003 + case["len_hi"] * 101 + case["new_hi"])
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(case["seqs"])]
    length = [_spread(rng, max(1, case["len_lo"]), case["len_hi"]) for _ in range(case["seqs"])]
    return new, [max(a, b) for a, b in zip(new, length)]


def _frequencies(rot, scaling):
    """Turns of each pair per position, and the factor on its values: base 10000, stretched by 8 from a length of 4096."""
    i = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    turns = torch.exp(-(2.0 * i / rot) * math.log(10000.0)) / (2.0 * math.pi)
    if scaling == "linear":
        return turns / 8.0, 1.0
    if scaling == "parts":                   # pairs of many turns in the old length stay, slow ones are stretched
        keep = ((turns * 4096.0 - 1.0) / 31.0).clamp(0.0, 1.0)
        return turns * (keep + (1.0 - keep) / 8.0), 0.1 * math.log(8.0) + 1.0
    return turns, 1.0


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    t = _TYPES[case["type"]]
    state = {"case": dict(case)}
    if "rot" in case:
        state["turns"], state["amplitude"] = _frequencies(case["rot"], case["scaling"])
    if case["op"] == "rotary":
        state["x"] = torch.randn(case["n"], case["heads"], case["dim"], generator=g, device="cuda").to(t)
        start = torch.randint(0, case["far"], (1,), generator=g, device="cuda")
        state["pos"] = ((start + torch.arange(case["n"], device="cuda") * max(1, case["far"] // case["n"])) % case["far"]).to(torch.int32)
        return state
    heads, kv, dim, page, seqs = (case[k] for k in ("heads", "kv", "dim", "page", "seqs"))
    new, length = _lengths(case)
    pages = [-(-a // page) for a in length]
    n = sum(new)
    state["n"], state["new"], state["length"] = n, new, length
    state["most_new"], state["most_length"] = max(new), max(length)
    off = [0]
    for a in new:
        off.append(off[-1] + a)
    state["q_off"] = torch.tensor(off, dtype=torch.int32, device="cuda")
    state["seq_len"] = torch.tensor(length, dtype=torch.int32, device="cuda")
    total = sum(pages) + 3                   # a cache serves others too: its pages are in no order
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    at, used = torch.zeros(seqs, max(pages), dtype=torch.int64), 0
    for s, a in enumerate(pages):
        at[s, :a] = torch.arange(used, used + a)
        used += a
    state["table"] = order[at.cuda()].contiguous()
    for name in ("k_pages", "v_pages"):
        shape = (total, kv, page, dim) if case["heads_first"] else (total, page, kv, dim)
        cache = torch.empty(shape, dtype=t, device="cuda")
        for part in cache.split(max(1, (1 << 27) // (page * kv * dim))):
            part.copy_(torch.randn(part.shape, generator=g, device="cuda"))
        state[name] = cache.transpose(1, 2) if case["heads_first"] else cache
    fused = torch.randn(n, heads + 2 * kv, dim, generator=g, device="cuda")
    if case["op"] == "attend":
        state["q"] = (fused[:, :heads] * 2.0).to(t).contiguous()
    else:                                    # as the projection leaves them: q, k and v of a token side by side
        fused = fused.to(t)
        state["q"], state["k"], state["v"] = fused[:, :heads], fused[:, heads:heads + kv], fused[:, heads + kv:]
    return state


def _rotate(x, pos, turns, amplitude, layout, inverse):
    """amplitude R(pos) x in fp32; angles in 64 bits, as a part of a turn."""
    part = pos.double()[:, None] * turns
    angle = (part - torch.round(part)) * (2.0 * math.pi)
    c, s = torch.cos(angle).float()[:, None] * amplitude, torch.sin(angle).float()[:, None] * amplitude
    if inverse:
        s = -s
    m = turns.numel()
    x = x.float()
    a, b = (x[..., :m], x[..., m:2 * m]) if layout == "half" else (x[..., 0:2 * m:2], x[..., 1:2 * m:2])
    u, w = a * c - b * s, b * c + a * s
    turned = torch.cat([u, w], -1) if layout == "half" else torch.stack([u, w], -1).flatten(-2)
    return torch.cat([turned, x[..., 2 * m:]], -1)


def _rows(state):
    """Of each row of new tokens: its sequence and its position in it."""
    q_off, n = state["q_off"].long(), state["n"]
    seq = torch.repeat_interleave(torch.arange(q_off.numel() - 1, device="cuda"), q_off[1:] - q_off[:-1], output_size=n)
    row = torch.arange(n, device="cuda")
    return seq, row - q_off[seq + 1] + state["seq_len"].long()[seq]


def _plain(state):
    case = state["case"]
    if case["op"] == "rotary":
        x = state["x"]
        return {"out": _rotate(x, state["pos"], state["turns"], state["amplitude"], case["layout"], case["inverse"]).to(x.dtype)}
    seq, pos = _rows(state)
    page, table = case["page"], state["table"].long()
    if case["op"] == "append":
        turn = lambda x: _rotate(x, pos, state["turns"], state["amplitude"], case["layout"], False).to(x.dtype)
        where = table[seq, pos // page], pos % page
        state["k_pages"][where] = turn(state["k"])
        state["v_pages"][where] = state["v"]
        return {"q": turn(state["q"]), "k_pages": state["k_pages"], "v_pages": state["v_pages"]}
    heads, kv, dim, seqs = case["heads"], case["kv"], case["dim"], case["seqs"]
    group, most, new = heads // kv, state["most_length"], state["most_new"]
    key = torch.arange(most, device="cuda")
    inside = key < state["seq_len"].long()[:, None]
    where = torch.where(inside, table[:, key // page], 0), (key % page).expand(seqs, most)
    k, v = state["k_pages"][where].float(), state["v_pages"][where].float()         # [seqs, most, kv, dim]
    row = torch.arange(state["n"], device="cuda") - state["q_off"].long()[seq]
    q = torch.zeros(seqs, new, kv, group, dim, device="cuda")
    q[seq, row] = state["q"].float().view(-1, kv, group, dim)
    at = torch.full((seqs, new), -1, dtype=torch.int64, device="cuda")
    at[seq, row] = pos
    seen = key <= at[..., None]                                                      # [seqs, new, most]
    if case["window"]:
        seen &= (key > at[..., None] - case["window"]) | (key < case["sinks"])
    z = q.permute(0, 2, 1, 3, 4).reshape(seqs, kv, new * group, dim) @ k.permute(0, 2, 3, 1)
    z = z.view(seqs, kv, new, group, most).mul_(dim ** -0.5)
    z.masked_fill_(~seen[:, None, :, None], float("-inf"))
    top = z.amax(-1, keepdim=True).clamp(min=-1e30)
    p = z.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = p.view(seqs, kv, new * group, most) @ v.permute(0, 2, 1, 3)
    o = o.view(seqs, kv, new, group, dim) / total
    lse = (top + torch.log(total))[..., 0]
    out = o.permute(0, 2, 1, 3, 4)[seq, row].reshape(-1, heads, dim).to(state["q"].dtype)
    return {"out": out, "lse": lse.permute(0, 2, 1, 3)[seq, row].reshape(-1, heads)}


def _own(state):
    from paper_2605_16154_b200 import binding as lib
    case = state["case"]
    interleaved = case.get("layout") == "interleaved"
    if case["op"] == "rotary":
        return {"out": lib.grpo_rotary(state["x"], state["pos"], state["turns"], interleaved=interleaved, amplitude=state["amplitude"],
                                       inverse=case["inverse"])}
    if case["op"] == "append":
        q = lib.grpo_rotary_cache(state["q"], state["k"], state["v"], state["k_pages"], state["v_pages"], state["table"], state["seq_len"],
                                  state["q_off"], state["turns"], interleaved=interleaved, amplitude=state["amplitude"])
        return {"q": q, "k_pages": state["k_pages"], "v_pages": state["v_pages"]}
    out, lse = lib.grpo_paged_attention(state["q"], state["k_pages"], state["v_pages"], state["table"], state["seq_len"], state["q_off"],
                                        window=case["window"], sinks=case["sinks"], max_new=state["most_new"])
    return {"out": out, "lse": lse}


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    """Each input read once, each output written once; of the cache what some row sees."""
    size = 4 if case["type"] == "f32" else 2
    if case["op"] == "rotary":
        count = case["n"] * case["heads"] * case["dim"]
        return {"bytes": 2 * count * size + 4 * case["n"], "flops": 3 * case["n"] * case["heads"] * case["rot"]}
    new, length = _lengths(case)
    heads, kv, dim = case["heads"], case["kv"], case["dim"]
    if case["op"] == "append":
        return {"bytes": 2 * sum(new) * (heads + 2 * kv) * dim * size, "flops": 3 * sum(new) * (heads + kv) * case["rot"]}
    window, sinks = case["window"], case["sinks"]
    read = pairs = 0
    for a, b in zip(new, length):
        first = b - a                        # position of the first new token
        if not window:
            read += b
            pairs += a * (first + 1 + b) // 2
            continue
        low = max(0, first - window + 1)
        read += b - low + min(sinks, low)
        for p in range(first, b):
            low = max(0, p - window + 1)
            pairs += p + 1 - low + min(sinks, low)
    return {"bytes": 2 * read * kv * dim * size + 2 * sum(new) * heads * dim * size + 4 * sum(new) * heads, "flops": 4 * pairs * heads * dim}


def _exact_turn(x, pos, case):
    """The rotation as products of complex numbers, its frequencies from the definition."""
    rot = case["rot"]
    inv = torch.tensor([10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)], dtype=torch.float64, device="cuda")
    amplitude = 1.0
    if case["scaling"] == "linear":
        pos = pos.double() / 8.0
    elif case["scaling"] == "parts":
        full = 4096.0 * inv / (2.0 * math.pi)
        share = torch.where(full < 1.0, 0.0, torch.where(full > 32.0, 1.0, (full - 1.0) / 31.0))
        inv = (1.0 - share) * inv / 8.0 + share * inv
        amplitude = 1.0 + 0.1 * math.log(8.0)
    angle = pos.double()[:, None] * inv
    if case.get("inverse"):
        angle = -angle
    unit = torch.polar(torch.full_like(angle, amplitude), angle)[:, None]
    x = x.double()
    front = x[..., :rot]
    pair = front.unflatten(-1, (2, rot // 2)).transpose(-1, -2) if case["layout"] == "half" else front.unflatten(-1, (rot // 2, 2))
    y = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * unit)
    y = y.transpose(-1, -2).flatten(-2) if case["layout"] == "half" else y.flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def exact(case, seed):
    """The definitions in 64 bits, one sequence at a time."""
    state = prepare(case, seed)
    if case["op"] == "rotary":
        return {"out": _exact_turn(state["x"], state["pos"], case)}
    page, table, new, length = case["page"], state["table"].long(), state["new"], state["length"]
    if case["op"] == "append":
        k, v = state["k_pages"].double(), state["v_pages"].double()
        q, row = [], 0
        for s, (a, b) in enumerate(zip(new, length)):
            pos = torch.arange(b - a, b, device="cuda")
            at, slot = table[s][pos // page], pos % page
            k[at, slot] = _exact_turn(state["k"][row:row + a], pos, case)
            v[at, slot] = state["v"][row:row + a].double()
            q.append(_exact_turn(state["q"][row:row + a], pos, case))
            row += a
        return {"q": torch.cat(q), "k_pages": k, "v_pages": v}
    heads, kv, dim = case["heads"], case["kv"], case["dim"]
    group = heads // kv
    out, lse, row = [], [], 0
    for s, (a, b) in enumerate(zip(new, length)):
        used = table[s, :-(-b // page)]
        k = state["k_pages"][used].flatten(0, 1)[:b].double()
        v = state["v_pages"][used].flatten(0, 1)[:b].double()
        q = state["q"][row:row + a].double()
        pos = torch.arange(b - a, b, device="cuda")[:, None]
        key = torch.arange(b, device="cuda")[None]
        hidden = key > pos
        if case["window"]:
            hidden = hidden | ((key <= pos - case["window"]) & (key >= case["sinks"]))
        o, ls = torch.empty(a, heads, dim, dtype=torch.float64, device="cuda"), torch.empty(a, heads, dtype=torch.float64, device="cuda")
        for c in range(kv):
            z = torch.einsum("ahd,bd->hab", q[:, c * group:(c + 1) * group], k[:, c]) / math.sqrt(dim)
            z = z.masked_fill(hidden, float("-inf"))
            total = torch.logsumexp(z, -1, keepdim=True)
            o[:, c * group:(c + 1) * group] = torch.einsum("hab,bd->ahd", torch.exp(z - total), v[:, c])
            ls[:, c * group:(c + 1) * group] = total[..., 0].t()
        out.append(o)
        lse.append(ls)
        row += a
    return {"out": torch.cat(out), "lse": torch.cat(lse)}
