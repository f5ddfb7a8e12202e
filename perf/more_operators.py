"""Products with 4-bit weights and the choice of a token, whose time is watched: through the public entry points.

A case names one pass.  The kinds:

  linear   dip_grouped_product with one 4-bit matrix: bfloat16 rows as they come, from one token to a prompt, and the head
           (binary32 logits)
  product  dip_grouped_product: a ragged group of rows per expert against that expert's 4-bit matrix
  mlp      dip_route_experts + dip_expert_mlp with 4-bit weights; top_k = 0 is the dense block of one expert that a prompt goes
           through, without a router
  sample   dip_sample_tokens: from logits, each row's temperature, top-k, top-p and min-p and one given number to a token and
           its probability

Weights are two codes a byte (even input index in the low nibble) along d_in, with a binary16 scale for each 128 inputs of
each output, [d_in / 128][d_out]: value = (code - 8) * scale.  Inputs are synthetic: N(0, 0.02) weights, heavy-tailed
activations, logits with a few favoured tokens.
"""
import math

import torch

own = False
GROUP = 128


def _linear(tokens, d_in, d_out, out="bf16", name=None):
    return _named({"kind": "linear", "tokens": tokens, "d_in": d_in, "d_out": d_out, "out": out}, name)


def _product(rows, experts, d_in, d_out, out="bf16", name=None):
    return _named({"kind": "product", "rows": rows, "experts": experts, "d_in": d_in, "d_out": d_out, "out": out}, name)


def _mlp(tokens, experts, top_k, d_model, d_ff, name=None):
    return _named({"kind": "mlp", "tokens": tokens, "experts": experts, "top_k": top_k, "d_model": d_model, "d_ff": d_ff}, name)


def _sample(rows, vocab, logits="f32", mode="mixed", masked=0.0, pad=0.0, name=None):
    return _named({"kind": "sample", "rows": rows, "vocab": vocab, "logits": logits, "mode": mode, "masked": masked, "pad": pad}, name)


def _named(c, name):
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token through one matrix of a decode loop: bound by the codes' bytes
        _linear(1, 5120, 17920, name="linear_token"),
        # the head of a decode step for eight sequences: logits for a large vocabulary
        _linear(8, 4096, 102400, "f32", name="linear_head"),
        # a small batch, sizes that are no multiple of a group
        _linear(77, 2080, 1056, name="linear_ragged"),
        # a long prompt through one matrix: bound by the tensor cores
        _linear(8192, 5120, 17920, name="linear_prompt"),
        # a short prompt over small experts of odd sizes, some of them empty
        _product(1531, 16, 1056, 2080, name="product_ragged"),
        # a decode step of a mixture: 2 of 8 experts for one token
        _mlp(1, 8, 2, 4096, 14336, name="mlp_token"),
        # a decode step of 16 sequences over many small experts: nearly all of them are read for a row or two
        _mlp(16, 64, 8, 1024, 2816, name="mlp_batch"),
        # a prompt through the dense block of a model whose decode is pruned
        _mlp(2048, 1, 0, 4096, 14336, name="mlp_dense_prompt"),
        # one sequence's next token, top-k and top-p together: latency
        _sample(1, 32064, "bf16", "top_kp", name="sample_token"),
        # a batch of requests, each with settings of its own, some tokens closed by a grammar, some rows unused
        _sample(64, 102400, "f32", "mixed", 0.2, 0.1, name="sample_batch"),
        # many sequences, a vocabulary of an odd size, top-p alone: the whole row counts
        _sample(512, 151001, "bf16", "top_p", name="sample_top_p"),
        # many sequences with a temperature only
        _sample(256, 50257, "f32", "plain", name="sample_plain"),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    """A case of the same kinds and ranges: 1 .. 8192 tokens or rows, 1 .. 128 experts, inputs of 256 .. 17920, outputs of
    64 .. 102400; 1 .. 512 rows of 1000 .. 160000 logits."""
    while True:
        kind = rng.choice(["linear", "linear", "product", "mlp", "mlp", "sample", "sample", "sample"])
        if kind == "sample":
            c = _sample(int(_log(rng, 1, 512.99)), int(_log(rng, 1000, 160000)), rng.choice(["f32", "bf16"]),
                        rng.choice(["mixed", "mixed", "top_kp", "top_k", "top_p", "min_p", "plain", "greedy"]),
                        rng.choice([0.0, 0.0, 0.3]), rng.choice([0.0, 0.0, 0.2]))
            if c["rows"] * c["vocab"] <= 512 * 151001:
                return c
            continue
        tokens = int(_log(rng, 1, 8192.99))
        experts = rng.choice([4, 8, 12, 16, 32, 60, 64, 100, 128])
        top_k = min(experts, rng.choice([1, 2, 2, 4, 6, 8]))
        d = int(_log(rng, 256, 5120)) // 32 * 32
        f = int(d * rng.uniform(0.3, 3.6)) // 32 * 32
        out = rng.choice(["bf16", "bf16", "f32"])
        if kind == "product":
            c = _product(tokens, experts, *rng.choice([(d, f), (f, d)]), out)
        elif kind == "linear":
            if rng.random() < 0.25:
                f = int(_log(rng, 32000, 102400)) // 32 * 32
                c = _linear(min(tokens, 256), d, f, "f32")
            else:
                c = _linear(tokens, *rng.choice([(d, f), (f, d)]), out)
        elif rng.random() < 0.3:
            c = _mlp(tokens, 1, 0, d, f)
        else:
            c = _mlp(tokens, experts, top_k, d, f)
        w = work(c)
        if 64 <= f <= 102400 and _weight_count(c) <= 1.4e9 and w["flops"] <= 1.5e12 and w["bytes"] <= 1e9:
            return c


def _weight_count(c):
    if c["kind"] == "mlp":
        return 3.0 * c["experts"] * c["d_model"] * c["d_ff"]
    return float(c.get("experts", 1)) * c["d_in"] * c["d_out"]


# ---- inputs ------------------------------------------------------------------------------------------------------------
def _groups_of(d):
    return -(-d // GROUP)


def _matrix(gen, experts, d_out, d_in):
    """[experts, d_out, d_in / 2] bytes of codes and [experts, ceil(d_in / 128), d_out] binary16 scales."""
    codes = torch.empty((experts, d_out, d_in // 2), device="cuda", dtype=torch.uint8)
    scales = torch.empty((experts, _groups_of(d_in), d_out), device="cuda", dtype=torch.float16)
    for e in range(experts):
        z = torch.randn((d_out, d_in), generator=gen, device="cuda").mul_(0.02)
        z = torch.nn.functional.pad(z, (0, -d_in % GROUP)).view(d_out, -1, GROUP)
        s = (z.abs().amax(dim=2) / 7.0).half()
        q = (z / s.float()[:, :, None]).round_().clamp_(-8, 7).add_(8).view(d_out, -1)[:, :d_in].to(torch.uint8)
        codes[e] = q[:, ::2] | (q[:, 1::2] << 4)
        scales[e] = s.t()
    return codes, scales


def _activations(gen, n, d):
    """Student-t(3) of unit rms: few large values, a broad middle."""
    v = torch.randn((n, d), generator=gen, device="cuda")
    chi = sum(torch.randn((n, d), generator=gen, device="cuda").square_() for _ in range(3)).div_(3)
    v = v / chi.sqrt().clamp_min(0.05)
    return (v / v.square().mean(dim=-1, keepdim=True).sqrt()).bfloat16()


def _vocabulary(gen, c):
    """Logits as a head leaves them: a broad middle, some twenty tokens that stand out by up to a dozen; tokens that a grammar
    closes (-inf, or the type's lowest value), rows without an open token."""
    n, v = c["rows"], c["vocab"]
    z = torch.randn((n, v), generator=gen, device="cuda").mul_(2.0)
    at = torch.randint(0, v, (n, 20), generator=gen, device="cuda")
    z.scatter_add_(1, at, 12.0 * torch.rand((n, 20), generator=gen, device="cuda"))
    z = z.bfloat16() if c["logits"] == "bf16" else z
    if c["masked"]:
        closed = torch.rand((n, v), generator=gen, device="cuda") < c["masked"]
        z[::2].masked_fill_(closed[::2], -math.inf)
        z[1::2].masked_fill_(closed[1::2], torch.finfo(z.dtype).min)
    if c["pad"]:
        z.masked_fill_(torch.rand((n, 1), generator=gen, device="cuda") < c["pad"], -math.inf)
    return z


def _settings(gen, c):
    """Each row's settings; None where the whole batch goes without."""
    n, mode = c["rows"], c["mode"]
    pick = lambda values, dtype=torch.float32: torch.tensor(values, device="cuda", dtype=dtype)[  # noqa: E731
        torch.randint(0, len(values), (n,), generator=gen, device="cuda")]
    s = {"temperature": 0.5 + torch.rand((n,), generator=gen, device="cuda"), "top_k": None, "top_p": None, "min_p": None}
    if mode == "greedy":
        s["temperature"] = torch.zeros((n,), device="cuda")
    if mode == "mixed":
        s["temperature"] *= pick([0.0, 1.0, 1.0, 1.0])
    if mode in ("top_k", "top_kp"):
        s["top_k"] = pick([20, 50, 200, 1000], torch.int32)
    if mode in ("top_p", "top_kp"):
        s["top_p"] = pick([0.5, 0.8, 0.9, 0.95])
    if mode == "min_p":
        s["min_p"] = pick([0.02, 0.05, 0.1])
    if mode == "mixed":
        s["top_k"], s["top_p"], s["min_p"] = pick([0, 0, 1, 40, 500], torch.int32), pick([1.0, 1.0, 0.5, 0.9, 0.99]), pick([0.0, 0.0, 0.05])
    return s


def _logits(gen, c):
    return torch.randn((c["tokens"], c["experts"]), generator=gen, device="cuda") + \
        0.7 * torch.randn((1, c["experts"]), generator=gen, device="cuda")


def _inputs(c, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": c}
    if c["kind"] == "sample":
        s["logits"] = _vocabulary(gen, c)
        s["settings"] = _settings(gen, c)
        s["uniform"] = torch.rand((c["rows"],), generator=gen, device="cuda")
    elif c["kind"] == "product":
        # rows of each expert as a router would leave them: favoured experts, every eighth without a row
        p = torch.softmax(0.5 * torch.randn(c["experts"], generator=gen, device="cuda"), 0)
        p[7::8] = 0
        e = torch.multinomial(p, c["rows"], replacement=True, generator=gen).sort().values.int()
        s["row_expert"] = e
        s["offset"] = torch.searchsorted(e, torch.arange(c["experts"] + 1, device="cuda", dtype=torch.int32)).int()
        s["x"] = _activations(gen, c["rows"], c["d_in"])
        s["w"] = _matrix(gen, c["experts"], c["d_out"], c["d_in"])
    elif c["kind"] == "linear":
        s["x"] = _activations(gen, c["tokens"], c["d_in"])
        s["w"] = _matrix(gen, 1, c["d_out"], c["d_in"])
    else:
        if c["top_k"]:
            s["logits"] = _logits(gen, c)
        s["x"] = _activations(gen, c["tokens"], c["d_model"])
        s["gate"] = _matrix(gen, c["experts"], c["d_ff"], c["d_model"])
        s["up"] = _matrix(gen, c["experts"], c["d_ff"], c["d_model"])
        s["down"] = _matrix(gen, c["experts"], c["d_model"], c["d_ff"])
    return s


_context = None


def prepare(case, seed):
    s = _inputs(case, seed)
    c = case
    # the most rows that one expert has: what a program that pads its groups keeps as their size
    if c["kind"] == "product":
        s["most"] = int((s["offset"][1:] - s["offset"][:-1]).max())
    elif c["kind"] == "mlp" and c["top_k"]:
        s["most"] = int(torch.bincount(s["logits"].topk(c["top_k"], dim=1).indices.flatten()).max())
    if own:
        import paper_2412_01380_b200 as dip

        global _context
        if _context is None:
            _context = dip.Context(torch.cuda.current_device())
        s["dip"] = dip
        if c["kind"] == "sample":
            s["token"] = torch.empty((c["rows"],), device="cuda", dtype=torch.int32)
            s["prob"] = torch.empty((c["rows"],), device="cuda")
        elif c["kind"] == "mlp":
            if c["top_k"]:
                s["route"] = dip.ExpertRoute(c["tokens"], c["experts"], c["top_k"], "cuda")
            s["weights"] = dip.ExpertWeights(*(dip.GroupedMatrix(*s[n]) for n in ("gate", "up", "down")))
            s["buffers"] = dip.ExpertWork(c["tokens"], c["top_k"], s["weights"], "cuda")
            s["y"] = torch.empty((c["tokens"], c["d_model"]), device="cuda", dtype=torch.bfloat16)
        else:
            s["rows"] = dip.Rows.of(s["x"])
            s["matrix"] = dip.GroupedMatrix(*s["w"])
            s["y"] = torch.empty((s["x"].shape[0], c["d_out"]), device="cuda",
                                 dtype=torch.bfloat16 if c["out"] == "bf16" else torch.float32)
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------------------
def _weight_values(codes, scales):
    """[n, d_out, d_in / 2], [n, groups, d_out] -> [n, d_out, d_in] binary32 (exact: 4 bits times 11)."""
    n, d_out, half = codes.shape
    q = torch.stack((codes & 15, codes >> 4), dim=3).view(n, d_out, 2 * half)
    s = scales.float().transpose(1, 2).repeat_interleave(GROUP, dim=2)[:, :, :2 * half]
    return (q.float() - 8.0) * s


def _choice(logits, top_k):
    """Each token's experts and weights."""
    expert = torch.argsort(logits, dim=1, descending=True, stable=True)[:, :top_k]
    part = torch.exp(logits.gather(1, expert) - logits.amax(dim=1, keepdim=True))
    return expert, part / part.sum(dim=1, keepdim=True)


def _groups(expert, experts):
    """The rows grouped by expert: each expert's first row, each row's token, each choice's row."""
    tokens, top_k = expert.shape
    order = torch.argsort(expert.flatten(), stable=True)
    offset = torch.searchsorted(expert.flatten()[order], torch.arange(experts + 1, device=expert.device))
    rank = torch.arange(tokens * top_k, device=expert.device)
    row = torch.empty_like(order).scatter_(0, order, rank)
    return offset, order // top_k, row.view(tokens, top_k)


def _grouped(values, row_expert, place, most, *matrices):
    """values[r] @ W[row_expert[r]].T for each matrix: few rows with a copy of their matrices, many in padded groups."""
    experts = matrices[0][0].shape[0]
    if values.shape[0] <= experts:
        return [torch.bmm(_weight_values(w[row_expert], s[row_expert]), values[:, :, None])[:, :, 0] for w, s in matrices]
    slot = row_expert * most + place
    padded = torch.zeros((experts * most, values.shape[1]), device=values.device).index_copy_(0, slot, values)
    padded = padded.view(experts, most, -1)
    return [torch.bmm(padded, _weight_values(w, s).transpose(1, 2)).view(experts * most, -1)[slot] for w, s in matrices]


def _silu(v):
    return v / (1 + torch.exp(-v))


def _drawn(logits, settings, uniform):
    """Each row's token and its probability, in 64 bits: whole rows in order of (logit descending, index ascending)."""
    z = logits.double()
    n, vocab = z.shape
    z = torch.where(torch.isnan(z), torch.full_like(z, -math.inf), z)
    high = z.amax(dim=1, keepdim=True)
    none = high == -math.inf
    t = settings["temperature"].double()[:, None]
    far = torch.where(z == high, torch.zeros_like(z), (z - torch.where(none, torch.zeros_like(high), high)) / torch.where(t > 0, t, torch.ones_like(t)))
    e = torch.where(none, torch.zeros_like(z), torch.exp(far))
    order = torch.argsort(z, dim=1, descending=True, stable=True)
    e = e.gather(1, order)
    rank = torch.arange(vocab, device=z.device)[None]
    keep = e > 0
    if settings["top_k"] is not None:
        k = settings["top_k"][:, None]
        keep &= (rank < k) | (k <= 0)
    if settings["top_p"] is not None:
        p = settings["top_p"].double()[:, None]
        mass = torch.where(keep, e, torch.zeros_like(e)).cumsum(dim=1)
        before = torch.cat((torch.zeros_like(mass[:, :1]), mass[:, :-1]), dim=1)
        keep &= (before < p * mass[:, -1:]) | (p >= 1)
    if settings["min_p"] is not None:
        keep &= e >= settings["min_p"].double()[:, None]
    keep &= (t > 0) | (rank == 0)
    e = torch.zeros_like(e).scatter_(1, order, torch.where(keep, e, torch.zeros_like(e)))
    mass = e.cumsum(dim=1)
    token = (mass <= uniform.double()[:, None] * mass[:, -1:]).sum(dim=1, keepdim=True).clamp_max(vocab - 1)
    prob = e.gather(1, token) / mass[:, -1:]
    token = torch.where(none, torch.full_like(token, -1), token)
    prob = torch.where(none, torch.zeros_like(prob), prob)
    return token[:, 0].int(), prob[:, 0].float()


def _plain(s):
    c = s["case"]
    if c["kind"] == "sample":
        token, prob = _drawn(s["logits"], s["settings"], s["uniform"])
        return {"token": token, "prob": prob}
    x = s["x"].float()
    if c["kind"] == "linear":
        y = x @ _weight_values(*s["w"])[0].t()
        return {"y": y.bfloat16() if c["out"] == "bf16" else y}
    if c["kind"] == "product":
        e = s["row_expert"].long()
        place = torch.arange(c["rows"], device=e.device) - s["offset"].long()[e]
        y = _grouped(x, e, place, s["most"], s["w"])[0]
        return {"y": y.bfloat16() if c["out"] == "bf16" else y}
    if not c["top_k"]:
        gate, up, down = (_weight_values(*s[n])[0].t() for n in ("gate", "up", "down"))
        return {"y": ((_silu(x @ gate) * (x @ up)) @ down).bfloat16()}
    expert, weight = _choice(s["logits"], c["top_k"])
    offset, row_token, row = _groups(expert, c["experts"])
    r = torch.arange(row_token.numel(), device=row.device)
    row_expert = torch.searchsorted(offset, r, right=True) - 1
    place = r - offset[row_expert]
    gate, up = _grouped(x[row_token], row_expert, place, s["most"], s["gate"], s["up"])
    out = _grouped(_silu(gate) * up, row_expert, place, s["most"], s["down"])[0]
    return {"y": (out[row] * weight[:, :, None]).sum(dim=1).bfloat16()}


# ---- one pass ----------------------------------------------------------------------------------------------------------
def _call(s):
    c, dip = s["case"], s["dip"]
    if c["kind"] == "sample":
        dip.dip_sample_tokens(_context, s["logits"], s["uniform"], s["token"], prob=s["prob"], **s["settings"])
        return {"token": s["token"], "prob": s["prob"]}
    if c["kind"] in ("linear", "product"):
        dip.dip_grouped_product(_context, s["matrix"], s["rows"], s["y"], offset=s.get("offset"))
    elif not c["top_k"]:
        dip.dip_expert_mlp(_context, s["weights"], s["x"], s["buffers"], s["y"])
    else:
        dip.dip_route_experts(_context, s["logits"], s["route"])
        dip.dip_expert_mlp(_context, s["weights"], s["x"], s["buffers"], s["y"], route=s["route"])
    return {"y": s["y"]}


def run(state):
    if own:
        return _call(state)
    return _plain(state)


# ---- what a pass cannot do without -------------------------------------------------------------------------------------
def _met(experts, choices):
    """Experts that meet a row when `choices` of them are made, all alike."""
    return experts * (1 - (1 - 1 / experts) ** choices) if experts > 1 else 1


def work(case):
    c = case
    if c["kind"] == "sample":
        n = float(c["rows"]) * c["vocab"]
        return {"bytes": n * (4.0 if c["logits"] == "f32" else 2.0) + 28.0 * c["rows"], "flops": 4.0 * n}
    item = 0.5 + 2.0 / GROUP                                                # (a weight, with its share of the scales)
    if c["kind"] in ("linear", "product"):
        rows = c["tokens"] if c["kind"] == "linear" else c["rows"]
        met = 1 if c["kind"] == "linear" else _met(c["experts"], rows)
        return {"bytes": met * c["d_in"] * c["d_out"] * item + rows * (2.0 * c["d_in"] + (2.0 if c["out"] == "bf16" else 4.0) * c["d_out"]),
                "flops": 2.0 * rows * c["d_in"] * c["d_out"]}
    rows = c["tokens"] * max(1, c["top_k"])
    met = c["experts"] * (1 - (1 - c["top_k"] / c["experts"]) ** c["tokens"]) if c["top_k"] else 1
    return {"bytes": met * 3 * c["d_model"] * c["d_ff"] * item + 4.0 * c["tokens"] * c["d_model"] + 4.0 * c["tokens"] * c["experts"],
            "flops": 6.0 * rows * c["d_model"] * c["d_ff"]}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------
def _matrix64(codes, scales, e):
    q, s = codes[e].double(), scales[e].double()
    high = (q / 16).floor_()
    w = torch.empty((q.shape[0], 2 * q.shape[1]), device="cuda", dtype=torch.float64)
    w[:, ::2], w[:, 1::2] = q - 16 * high, high
    w -= 8
    for g in range(s.shape[0]):
        w[:, g * GROUP:(g + 1) * GROUP] *= s[g][:, None]
    return w


def _probabilities64(z, u, temperature, top_k=0, top_p=1.0, min_p=0.0):
    """One row of binary64 logits: the probability of the token that u draws."""
    if not (z > -math.inf).any():
        return 0.0
    if not temperature > 0:
        return 1.0
    value, index = torch.sort(z, descending=True, stable=True)
    weight = torch.softmax((value - value[0]) / temperature, 0)
    count = min(top_k, weight.numel()) if top_k > 0 else weight.numel()
    weight = weight[:count] / weight[:count].sum()
    if top_p < 1:
        weight = weight[:1 + int((weight.cumsum(0)[:-1] < top_p).sum())]
    weight = weight[weight >= min_p * weight[0]]
    weight /= weight.sum()
    index, by_index = index[:weight.numel()].sort()
    place = torch.searchsorted(weight[by_index].cumsum(0), torch.full((1,), u, device=z.device, dtype=torch.float64), right=True)
    return float(weight[by_index][place.clamp_max(weight.numel() - 1)])


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    if c["kind"] == "sample":
        keep = {k: v.tolist() for k, v in s["settings"].items() if v is not None}
        prob = [_probabilities64(s["logits"][r].double(), u, **{k: v[r] for k, v in keep.items()})
                for r, u in enumerate(s["uniform"].tolist())]
        return {"token": None, "prob": torch.tensor(prob, device="cuda", dtype=torch.float64)}
    x = s["x"].double()
    if c["kind"] == "linear":
        return {"y": x @ _matrix64(*s["w"], 0).t()}
    if c["kind"] == "product":
        y = torch.zeros((c["rows"], c["d_out"]), device="cuda", dtype=torch.float64)
        for e, (a, b) in enumerate(zip(s["offset"].tolist()[:-1], s["offset"].tolist()[1:])):
            if b > a:
                y[a:b] = x[a:b] @ _matrix64(*s["w"], e).t()
        return {"y": y}
    if c["top_k"]:
        weight, expert = torch.sort(torch.softmax(s["logits"].double(), dim=1), dim=1, descending=True, stable=True)
        weight, expert = weight[:, :c["top_k"]] / weight[:, :c["top_k"]].sum(dim=1, keepdim=True), expert[:, :c["top_k"]]
    y = torch.zeros((c["tokens"], c["d_model"]), device="cuda", dtype=torch.float64)
    for e in range(c["experts"]):
        at = torch.arange(c["tokens"], device="cuda") if not c["top_k"] else (expert == e).any(dim=1).nonzero()[:, 0]
        if not at.numel():
            continue
        gate, up = (x[at] @ _matrix64(*s[n], e).t() for n in ("gate", "up"))
        out = (gate * torch.sigmoid(gate) * up) @ _matrix64(*s["down"], e).t()
        y[at] += out * (weight * (expert == e)).sum(dim=1, keepdim=True)[at] if c["top_k"] else out
    return {"y": y}
