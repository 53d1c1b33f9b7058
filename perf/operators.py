"""The operators of decoding in small numbers, as a list of timed cases: products with 4-bit weights, attention over source
rows held in 8 bits, and a beam search's choice with the states that follow it.

A case is one call as a decoder makes it.  `run` computes it in elementary torch operations, or, where `own` is true, with
the operators of paper_1802_07170_amd/decoding.py.  Shapes are those of the workloads in paper_1802_07170_amd/inputs.py
where it has one (hidden sizes 336 to 1024, vocabularies of 9064 to 50000, 10 beams, sentences of 3 to 120 tokens), and
generic otherwise (several heads, long documents)."""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda"
BLOCK = 32                                     # tokens that share a scale in the cache
MAGNITUDES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]      # of a 4-bit code's lower three bits; the fourth is the sign


def listed():
    return [
        # one sentence's next token: the gates of one layer of the 1024-wide decoder, [input; state] against [4H, 2H]
        dict(name="gates_one", kind="product", rows=1, outputs=4096, inputs=2048, group=64, dtype="bf16", out="fp32", bias=True, tanh=False),
        # the output layer for the 10 hypotheses of one sentence
        dict(name="logits_beam", kind="product", rows=10, outputs=32000, inputs=1024, group=64, dtype="bf16", out="fp32", bias=True, tanh=False),
        # the output layer of a whole batch's search: 64 sentences, 10 hypotheses each
        dict(name="logits_batch", kind="product", rows=640, outputs=32000, inputs=1024, group=128, dtype="bf16", out="fp32", bias=True, tanh=False),
        # the attentional layer in full precision at a width that is no round number: 23 greedy rows, tanh behind the product
        dict(name="tanh_ragged", kind="product", rows=23, outputs=336, inputs=672, group=32, dtype="fp32", out="fp32", bias=False, tanh=True),
        # one position of a search over one sentence: the choice among 10 x 32000, and the states of four layers behind it
        dict(name="search_one", kind="search", sentences=1, beam=10, vocab=32000, hidden=1024, layers=4, dtype="fp32"),
        # the same for a batch of 64 sentences
        dict(name="search_batch", kind="search", sentences=64, beam=10, vocab=32000, hidden=1024, layers=4, dtype="fp32"),
        # a narrow beam over an odd vocabulary, logits and states in 16 bits (equal logits are common there)
        dict(name="search_ragged", kind="search", sentences=23, beam=4, vocab=9064, hidden=336, layers=3, dtype="bf16"),
        # one position's attention of a batch's search: hypotheses of a sentence share its source rows
        dict(name="attend_beams", kind="attend", sequences=64, per=10, heads=1, kv_heads=1, dim=1024, lo=20, hi=50, dtype="bf16"),
        # one sentence as it arrives, in full precision
        dict(name="attend_one", kind="attend", sequences=1, per=10, heads=1, kv_heads=1, dim=512, lo=25, hi=25, dtype="fp32"),
        # long documents, several heads that share keys and values, one query each
        dict(name="attend_documents", kind="attend", sequences=8, per=1, heads=16, kv_heads=4, dim=128, lo=8000, hi=32768, dtype="bf16"),
        # the source rows of a large batch, written once before its search
        dict(name="fill_batch", kind="fill", sequences=128, kv_heads=1, dim=1024, lo=30, hi=80, dtype="bf16"),
        # uneven sentences of an odd width in full precision
        dict(name="fill_ragged", kind="fill", sequences=23, kv_heads=1, dim=336, lo=3, hi=37, dtype="fp32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 6e12, w["flops"] / 4e14)


def draw(rng):
    """One more case: 1 to 640 rows, widths of 16 to 4096, vocabularies of 1000 to 50000, 1 to 128 sentences, sources of one token to
    32768, heads of 16 to 1024.  What is most numerous is halved until the case costs no more than the largest listed one."""
    kind = rng.choice(["product", "product", "search", "attend", "attend", "fill"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if kind == "product":
        case = dict(kind=kind, rows=_log_int(rng, 1, 640), outputs=_log_int(rng, 16, 50000), inputs=_log_int(rng, 16, 4096),
                    group=rng.choice([32, 64, 128]), dtype=dtype, out=rng.choice(["fp32", dtype]), bias=rng.random() < 0.7, tanh=rng.random() < 0.3)
        shrink = "rows"
    elif kind == "search":
        case = dict(kind=kind, sentences=_log_int(rng, 1, 64), beam=rng.randint(1, 16), vocab=_log_int(rng, 1000, 50000),
                    hidden=16 * _log_int(rng, 1, 64), layers=rng.randint(1, 4), dtype=dtype)
        shrink = "sentences"
    else:
        kv = rng.choice([1, 1, 2, 4])
        hi = _log_int(rng, 1, 32768)
        case = dict(kind=kind, sequences=_log_int(rng, 1, 128), kv_heads=kv, dim=16 * _log_int(rng, 1, 64 // kv), lo=rng.randint(max(1, hi // 5), hi),
                    hi=hi, dtype=dtype)
        if kind == "attend":
            case |= dict(per=rng.randint(1, 16) if kv == 1 else 1, heads=kv * rng.choice([1, 2, 4]))
        shrink = "sequences"
    most = max(_cost(c) for c in listed() if c["kind"] == kind)
    while case[shrink] > 1 and _cost(case) > most:
        case[shrink] //= 2
    while kind in ("attend", "fill") and case["hi"] > 1 and _cost(case) > most:
        case["hi"] //= 2
        case["lo"] = min(case["lo"], case["hi"])
    return case


def _type(name):
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[name]


def _random(seed):
    """Draws on the GPU from the seed alone."""
    generator = torch.Generator(device=DEVICE).manual_seed(seed)
    return lambda *shape: torch.randn(*shape, generator=generator, device=DEVICE)


def _inputs(case, seed):
    """What a decoder has in hand before the call."""
    randn, dtype = _random(seed), _type(case["dtype"])
    if case["kind"] == "product":
        m, n, k, g = case["rows"], case["outputs"], case["inputs"], case["group"]
        groups = -(-k // g)
        weight = torch.zeros(n, groups * g, device=DEVICE)             # trained weights, with rows of different sizes
        weight[:, :k] = randn(n, k) * (0.03 * torch.exp(0.3 * randn(n, 1)))
        by_group = weight.view(n, groups, g)
        scales = (by_group.abs().amax(2) / 6).to(torch.bfloat16)
        size = by_group.abs() / scales.float().clamp_min(1e-30)[:, :, None]
        code = torch.zeros_like(size, dtype=torch.uint8)
        for low in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0):
            code += size > low
        codes = (code + 8 * (by_group < 0)).view(n, groups * g)[:, :k].contiguous()
        return dict(x=torch.tanh(randn(m, k)).to(dtype), codes=codes, scales=scales, bias=0.1 * randn(n) if case["bias"] else None)
    if case["kind"] == "search":
        b, beam, v, h = case["sentences"], case["beam"], case["vocab"], case["hidden"]
        prior = -1.1 * torch.log(torch.arange(1, v + 1, device=DEVICE).float())        # words are as frequent as in a text
        order = torch.argsort(randn(v))
        logits = (randn(b, beam, v) * 1.5 + prior[order]).view(b * beam, v).to(dtype)
        scores = -torch.cumsum(torch.rand(b, beam, generator=torch.Generator(device=DEVICE).manual_seed(seed + 1), device=DEVICE), 1) * 0.7 - 5.0
        ended = torch.arange(beam, device=DEVICE)[None] >= beam - torch.arange(b, device=DEVICE)[:, None] % 3 * (beam // 4)
        scores[ended] = -math.inf                                      # places of hypotheses that have ended
        wide = [torch.tanh(randn(b * beam, h)).to(_type("bf16") if case["dtype"] == "bf16" else torch.float32) for _ in range(case["layers"] + 1)]
        cells = [randn(b * beam, h) for _ in range(case["layers"])]
        return dict(logits=logits, scores=scores, states=wide + cells)
    b, s, kv, d = case["sequences"], case["hi"], case["kv_heads"], case["dim"]
    lengths = torch.randint(case["lo"], s + 1, (b,), generator=torch.Generator(device=DEVICE).manual_seed(seed + 1), device=DEVICE, dtype=torch.int32)
    keys = (randn(b, s, kv, d) * (2.0 / math.sqrt(d))).to(dtype)
    values = torch.tanh(randn(b, s, kv, d)).to(dtype)
    given = dict(keys=keys, values=values, lengths=lengths)
    if case["kind"] == "attend":
        given["q"] = torch.tanh(randn(b * case["per"], case["heads"], d)).to(dtype)
    return given


def _in_blocks(x, lengths):
    """Codes [b, s, heads, d] in whole numbers of -127 to 127 and scales [b, blocks, heads] of the valid tokens."""
    b, s, kv, d = x.shape
    blocks = -(-s // BLOCK)
    padded = torch.zeros(b, blocks * BLOCK, kv, d, device=x.device)
    padded[:, :s] = x.float()
    padded *= (torch.arange(blocks * BLOCK, device=x.device)[None] < lengths[:, None])[:, :, None, None]
    padded = padded.view(b, blocks, BLOCK, kv, d)
    # (the quotients in 64 bits: many of those of 16-bit values lie on the border between two codes, and the last bit of a scale moves them)
    scales = (padded.abs().amax((2, 4)).double() / 127).float()
    codes = torch.round(padded.double() / torch.where(scales > 0, scales, 1.0)[:, :, None, :, None].double()).to(torch.int8)
    return codes.view(b, blocks * BLOCK, kv, d)[:, :s], scales


def prepare(case, seed):
    """The inputs; weights and source rows in the form in which a decoder keeps them, made once."""
    state = dict(case=case, **_inputs(case, seed))
    kind = case["kind"]
    if kind in ("attend", "fill") and own:
        from paper_1802_07170_amd import decoding
        state["cache"] = decoding.SourceCache(case["sequences"], case["kv_heads"], case["dim"], case["hi"], device=state["keys"].device)
    if kind == "attend":
        if own:
            state["cache"].fill(state.pop("keys"), state.pop("values"), state["lengths"])
        else:
            state["keys"] = _in_blocks(state["keys"], state["lengths"])
            state["values"] = _in_blocks(state["values"], state["lengths"])
    if kind == "product" and own:
        from paper_1802_07170_amd import decoding
        state["weight"] = decoding.QuantWeight.from_codes(state.pop("codes").to(torch.uint8), state.pop("scales"), case["group"])
    if kind == "search":
        state["moved"] = [torch.zeros_like(t) for t in state["states"]]
    return state


def _product(case, s):
    table = torch.tensor(MAGNITUDES + [-v for v in MAGNITUDES], device=DEVICE)
    weight = table[s["codes"].long()] * s["scales"].float().repeat_interleave(case["group"], 1)[:, :case["inputs"]]
    y = s["x"].float() @ weight.T
    if s["bias"] is not None:
        y = y + s["bias"]
    return (torch.tanh(y) if case["tanh"] else y).to(_type(case["out"]))


def _search(case, s):
    """In 64 bits: which of two extensions is better may hang on the last bit.  The first of equal ones is taken."""
    b, beam, v = case["sentences"], case["beam"], case["vocab"]
    z = s["logits"].double().view(b, beam, v)
    top = z.amax(2, keepdim=True)
    all_scores = (s["scores"].double()[:, :, None] + z - top - torch.exp(z - top).sum(2, keepdim=True).log()).view(b, beam * v)
    best, scores = [], []
    for _ in range(beam):
        at = torch.argmax(all_scores, 1, keepdim=True)
        scores.append(all_scores.gather(1, at))
        best.append(at)
        all_scores.scatter_(1, at, -math.inf)
    scores, best = torch.cat(scores, 1), torch.cat(best, 1)
    found = scores > -math.inf
    rows = torch.where(found, best // v + beam * torch.arange(b, device=DEVICE)[:, None], -1).int()
    for old, new in zip(s["states"], s["moved"]):
        new.copy_(torch.where((rows >= 0).view(-1, 1), old[rows.view(-1).clamp_min(0)], new))
    return scores.float(), rows, torch.where(found, best % v, -1).int()


def _attend(case, s):
    b, per, heads, kv, d = case["sequences"], case["per"], case["heads"], case["kv_heads"], case["dim"]
    in_full = lambda t: t[0].float() * t[1].repeat_interleave(BLOCK, 1)[:, :t[0].shape[1], :, None]
    keys, values = in_full(s["keys"]).permute(0, 2, 1, 3).contiguous(), in_full(s["values"]).permute(0, 2, 1, 3).contiguous()
    q = s["q"].float().view(b, per, kv, heads // kv, d).permute(0, 2, 1, 3, 4).reshape(b, kv, per * (heads // kv), d)
    scores = q @ keys.transpose(2, 3).contiguous() / math.sqrt(d)
    hidden = torch.arange(keys.shape[2], device=DEVICE)[None] >= s["lengths"][:, None]
    scores = scores.masked_fill(hidden[:, None, None], -math.inf)
    weights = torch.exp(scores - scores.amax(3, keepdim=True))
    out = (weights @ values) / weights.sum(3, keepdim=True)
    return out.view(b, kv, per, heads // kv, d).permute(0, 2, 1, 3, 4).reshape(b * per, heads, d).to(_type(case["dtype"]))


def _fill(case, s):
    read = []
    for t in (s["keys"], s["values"]):
        codes, scales = _in_blocks(t, s["lengths"])
        read.append(codes.float() * scales.repeat_interleave(BLOCK, 1)[:, :codes.shape[1], :, None])
    return read


def run(state):
    case, kind = state["case"], state["case"]["kind"]
    if not own:
        if kind == "search":
            return [*_search(case, state), *state["moved"]]
        return {"product": _product, "attend": _attend, "fill": _fill}[kind](case, state)
    from paper_1802_07170_amd import decoding
    if kind == "product":
        return decoding.quant_product(state["x"], state["weight"], bias=state["bias"], tanh=case["tanh"], out_dtype=_type(case["out"]))
    if kind == "search":
        scores, rows, tokens = decoding.beam_select(state["logits"], state["scores"])
        decoding.beam_reorder(rows, state["states"], state["moved"])
        return [scores, rows, tokens, *state["moved"]]
    if kind == "attend":
        return state["cache"].attend(state["q"], scale=1.0 / math.sqrt(case["dim"]))
    state["cache"].fill(state["keys"], state["values"], state["lengths"])
    return list(state["cache"].read())


def exact(case, seed):
    """The definitions in 64 bits."""
    s, kind = _inputs(case, seed), case["kind"]
    if kind == "product":
        c = s["codes"].double()
        sign = torch.where(c >= 8, -1.0, 1.0).double()
        e = torch.remainder(c, 8)
        size = torch.where(e < 2, e * 0.5, (1 + 0.5 * torch.remainder(e, 2)) * torch.pow(torch.full_like(e, 2.0), torch.floor(e / 2) - 1))
        column = torch.arange(case["inputs"], device=DEVICE) // case["group"]
        y = torch.matmul(s["x"].double(), (sign * size * s["scales"].double()[:, column]).t())
        y = y + (0 if s["bias"] is None else s["bias"].double())
        return y.tanh() if case["tanh"] else y
    if kind == "search":
        b, beam, v = case["sentences"], case["beam"], case["vocab"]
        logp = torch.log_softmax(s["logits"].double().view(b, beam, v), 2) + s["scores"].double()[:, :, None]
        scores = torch.topk(logp.view(b, -1), beam, 1).values
        return [scores] + [None] * (2 + len(s["states"]))
    lengths = s["lengths"].tolist()
    held = {}
    for name in ("keys", "values"):
        x = s[name].double()
        for at, n in enumerate(lengths):
            x[at, n:] = 0
            for t in range(0, n, BLOCK):
                part = x[at, t:min(n, t + BLOCK)]
                unit = (part.abs().amax((0, 2), keepdim=True) / 127).float().double()
                unit[unit == 0] = 1
                part.copy_((part / unit).round() * unit)
        held[name] = x
    if kind == "fill":
        return [held["keys"], held["values"]]
    per, share = case["per"], case["heads"] // case["kv_heads"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEVICE)
    for r in range(s["q"].shape[0]):
        at = r // per
        for head in range(case["heads"]):
            k, v = held["keys"][at, :lengths[at], head // share], held["values"][at, :lengths[at], head // share]
            out[r, head] = torch.softmax(k @ s["q"][r, head].double() / math.sqrt(case["dim"]), 0) @ v
    return out


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "product":
        m, n, k = case["rows"], case["outputs"], case["inputs"]
        result = 2 if case["out"] == "bf16" else 4
        return {"bytes": n * k // 2 + 2 * n * -(-k // case["group"]) + m * k * size + m * n * result + (4 * n if case["bias"] else 0), "flops": 2 * m * n * k}
    if case["kind"] == "search":
        rows, v, h = case["sentences"] * case["beam"], case["vocab"], case["hidden"]
        states = 2 * rows * h * (size * (case["layers"] + 1) + 4 * case["layers"])
        return {"bytes": rows * v * size + states + 16 * rows, "flops": 4 * rows * v}
    tokens = case["sequences"] * (case["lo"] + case["hi"]) // 2 * case["kv_heads"]
    held = 2 * (tokens * case["dim"] + 4 * -(-tokens // BLOCK))
    if case["kind"] == "fill":
        return {"bytes": 2 * tokens * case["dim"] * size + held + 2 * case["sequences"] * case["hi"] * case["kv_heads"] * case["dim"] * 4,
                "flops": 8 * tokens * case["dim"]}
    queries = case["sequences"] * case["per"] * case["heads"]
    return {"bytes": held + 2 * queries * case["dim"] * size, "flops": 4 * queries * (case["lo"] + case["hi"]) // 2 * case["dim"]}
