"""The expert and dense SwiGLU products whose time is watched: what a serving loop asks of them, through the public entry points.

A case names one pass.  The kinds:

  route    dip_route_experts: from router logits to each token's experts and weights, and the rows grouped by expert
  product  dip_grouped_product: a ragged group of rows per expert against that expert's matrix, rows already in place
  linear   dip_grouped_product with one matrix, tokens as they come (8 bits: behind dip_stage_rows, which quantises them)
  mlp      dip_route_experts + dip_expert_mlp: logits and activations to the mixture's output; top_k = 0 is the dense
           block of one expert that a prompt goes through, without a router

Weights are [d_out, d_in], bfloat16 or e4m3 with a binary32 scale for each block of 128 x 128; 8-bit activations have a
binary32 scale for each token and 128 columns: max(amax / 448, 2^-126), codes rne(x / scale).  Activations and outputs
are bfloat16.  Inputs are synthetic: N(0, 0.02) weights, heavy-tailed activations, logits with favoured experts.
"""
import math

import torch

own = False
BLOCK = 128
TINY = 2.0 ** -126
TOP = 448.0


def _route(tokens, experts, top_k, logits="f32", renorm=True, pad=0.0, masked=0.0, name=None):
    return _named({"kind": "route", "tokens": tokens, "experts": experts, "top_k": top_k, "logits": logits, "renorm": renorm,
                   "pad": pad, "masked": masked}, name)


def _product(wtype, rows, experts, d_in, d_out, name=None):
    return _named({"kind": "product", "wtype": wtype, "rows": rows, "experts": experts, "d_in": d_in, "d_out": d_out}, name)


def _linear(wtype, tokens, d_in, d_out, name=None):
    return _named({"kind": "linear", "wtype": wtype, "tokens": tokens, "d_in": d_in, "d_out": d_out}, name)


def _mlp(wtype, tokens, experts, top_k, d_model, d_ff, name=None):
    return _named({"kind": "mlp", "wtype": wtype, "tokens": tokens, "experts": experts, "top_k": top_k, "d_model": d_model,
                   "d_ff": d_ff}, name)


def _named(c, name):
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of a decode loop picks 8 of 64 experts: latency
        _route(1, 64, 8, name="route_token"),
        # a packed batch of prompts, a tenth of it padding (no expert at all), a quarter of the experts closed to each token
        _route(16384, 128, 8, "bf16", False, 0.1, 0.25, name="route_prompt"),
        # one token's two experts: the smallest product with full-size matrices, bound by the weights' bytes
        _product("bf16", 2, 8, 4096, 14336, name="product_token"),
        # a short prompt over small experts of odd sizes, some of them empty
        _product("bf16", 1531, 16, 1056, 2080, name="product_ragged"),
        # a long prompt over many small experts: some hundred rows each
        _product("bf16", 16384, 64, 1024, 2816, name="product_prompt"),
        # one token through one 8-bit matrix: the weights are read once
        _linear("fp8", 1, 5120, 17920, name="fp8_token"),
        # a small batch, sizes that are no multiple of the block of 128
        _linear("fp8", 77, 2080, 1056, name="fp8_ragged"),
        # a long prompt through one 8-bit matrix: bound by the tensor cores
        _linear("fp8", 8192, 5120, 17920, name="fp8_prompt"),
        # a decode step of a mixture: 2 of 8 experts for one token
        _mlp("bf16", 1, 8, 2, 4096, 14336, name="mlp_token"),
        # its prompt
        _mlp("bf16", 4096, 8, 2, 4096, 14336, name="mlp_prompt"),
        # a decode step of 16 sequences over many small 8-bit experts: nearly all of them are read for a row or two
        _mlp("fp8", 16, 64, 8, 1024, 2816, name="mlp_fp8_batch"),
        # a prompt through the dense block of a model whose decode is pruned
        _mlp("fp8", 2048, 1, 0, 5120, 17920, name="mlp_fp8_dense_prompt"),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    """A case of the same kinds and ranges: 1 .. 16384 tokens or rows, 1 .. 128 experts, sizes of 256 .. 17920."""
    while True:
        kind = rng.choice(["route", "product", "product", "linear", "linear", "mlp", "mlp", "mlp"])
        tokens = int(_log(rng, 1, 16384.99))
        experts = rng.choice([4, 8, 12, 16, 32, 60, 64, 100, 128])
        top_k = min(experts, rng.choice([1, 2, 2, 4, 6, 8]))
        wtype = rng.choice(["bf16", "fp8"])
        d = int(_log(rng, 256, 5120)) // 32 * 32
        f = int(d * rng.uniform(0.3, 3.6)) // 32 * 32
        if kind == "route":
            return _route(tokens, experts, top_k, rng.choice(["f32", "bf16"]), rng.random() < 0.5,
                          rng.choice([0.0, 0.0, 0.2]), rng.choice([0.0, 0.0, 0.3]))
        if kind == "product":
            c = _product(wtype, tokens, experts, *rng.choice([(d, f), (f, d)]))
        elif kind == "linear":
            c = _linear(wtype, tokens, *rng.choice([(d, f), (f, d)]))
        elif rng.random() < 0.3:
            c = _mlp(wtype, tokens, 1, 0, d, f)
        else:
            c = _mlp(wtype, tokens, experts, top_k, d, f)
        w = work(c)
        if 64 <= f <= 17920 and _weight_count(c) <= 1.4e9 and w["flops"] <= 2.8e12 and w["bytes"] <= 2.8e9:
            return c


def _weight_count(c):
    if c["kind"] == "mlp":
        return 3.0 * c["experts"] * c["d_model"] * c["d_ff"]
    return float(c.get("experts", 1)) * c["d_in"] * c["d_out"]


# ---- inputs ------------------------------------------------------------------------------------------------------------
def _blocks(n):
    return -(-n // BLOCK)


def _matrix(gen, wtype, experts, d_out, d_in):
    """[experts, d_out, d_in] weights in their storage type, and the scales of the 128 x 128 blocks."""
    w = torch.empty((experts, d_out, d_in), device="cuda", dtype=torch.bfloat16 if wtype == "bf16" else torch.float8_e4m3fn)
    scales = None if wtype == "bf16" else torch.empty((experts, _blocks(d_out), _blocks(d_in)), device="cuda")
    for e in range(experts):
        z = torch.randn((d_out, d_in), generator=gen, device="cuda").mul_(0.02)
        if wtype == "bf16":
            w[e] = z
            continue
        b = torch.nn.functional.pad(z, (0, -d_in % BLOCK, 0, -d_out % BLOCK)).view(_blocks(d_out), BLOCK, _blocks(d_in), BLOCK)
        s = (b.abs().amax(dim=(1, 3)) / TOP).clamp_min(TINY)
        w[e] = (b / s[:, None, :, None]).reshape(b.shape[0] * BLOCK, -1)[:d_out, :d_in].to(torch.float8_e4m3fn)
        scales[e] = s
    return w, scales


def _activations(gen, n, d):
    """Student-t(3) of unit rms: few large values, a broad middle."""
    v = torch.randn((n, d), generator=gen, device="cuda")
    chi = sum(torch.randn((n, d), generator=gen, device="cuda").square_() for _ in range(3)).div_(3)
    v = v / chi.sqrt().clamp_min(0.05)
    return (v / v.square().mean(dim=-1, keepdim=True).sqrt()).bfloat16()


def _logits(gen, c):
    z = torch.randn((c["tokens"], c["experts"]), generator=gen, device="cuda")
    z += 0.7 * torch.randn((1, c["experts"]), generator=gen, device="cuda")
    if c.get("masked"):
        z.masked_fill_(torch.rand(z.shape, generator=gen, device="cuda") < c["masked"], -math.inf)
    if c.get("pad"):
        z.masked_fill_(torch.rand((c["tokens"], 1), generator=gen, device="cuda") < c["pad"], -math.inf)
    return z.bfloat16() if c.get("logits") == "bf16" else z


def _inputs(c, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": c}
    if c["kind"] == "route":
        s["logits"] = _logits(gen, c)
    elif c["kind"] == "product":
        # rows of each expert as a router would leave them: favoured experts, every eighth without a row
        p = torch.softmax(0.5 * torch.randn(c["experts"], generator=gen, device="cuda"), 0)
        p[7::8] = 0
        e = torch.multinomial(p, c["rows"], replacement=True, generator=gen).sort().values.int()
        s["row_expert"] = e
        s["offset"] = torch.searchsorted(e, torch.arange(c["experts"] + 1, device="cuda", dtype=torch.int32)).int()
        s["x"] = _activations(gen, c["rows"], c["d_in"])
        if c["wtype"] == "fp8":
            s["x"], s["x_scale"] = _codes(s["x"].float())
        s["w"] = _matrix(gen, c["wtype"], c["experts"], c["d_out"], c["d_in"])
    elif c["kind"] == "linear":
        s["x"] = _activations(gen, c["tokens"], c["d_in"])
        s["w"] = _matrix(gen, c["wtype"], 1, c["d_out"], c["d_in"])
    else:
        if c["top_k"]:
            s["logits"] = _logits(gen, c)
        s["x"] = _activations(gen, c["tokens"], c["d_model"])
        s["gate"] = _matrix(gen, c["wtype"], c["experts"], c["d_ff"], c["d_model"])
        s["up"] = _matrix(gen, c["wtype"], c["experts"], c["d_ff"], c["d_model"])
        s["down"] = _matrix(gen, c["wtype"], c["experts"], c["d_model"], c["d_ff"])
    return s


_context = None


def prepare(case, seed):
    s = _inputs(case, seed)
    c = case
    # the most rows that one expert has: what a program that pads its groups keeps as their size
    if c["kind"] == "product":
        s["most"] = int((s["offset"][1:] - s["offset"][:-1]).max())
    elif c["kind"] == "mlp" and c["top_k"]:
        s["most"] = int(torch.bincount(s["logits"].float().topk(c["top_k"], dim=1).indices.flatten()).max())
    if own:
        import paper_2412_01380_b200 as dip

        global _context
        if _context is None:
            _context = dip.Context(torch.cuda.current_device())
        s["dip"] = dip
        wtype = dip.W_BF16 if c.get("wtype") == "bf16" else dip.W_FP8_B128
        if c["kind"] in ("route", "mlp") and c["top_k"]:
            s["route"] = dip.ExpertRoute(c["tokens"], c["experts"], c["top_k"], "cuda")
        if c["kind"] == "product":
            s["rows"] = dip.Rows.of(s["x"], s.get("x_scale"))
        elif c["kind"] == "linear":
            s["rows"] = dip.Rows.of(s["x"]) if c["wtype"] == "bf16" else dip.Rows(c["tokens"], c["d_in"], wtype, "cuda")
        if c["kind"] in ("product", "linear"):
            s["matrix"] = dip.GroupedMatrix(*s["w"])
            s["y"] = torch.empty((s["x"].shape[0], c["d_out"]), device="cuda", dtype=torch.bfloat16)
        elif c["kind"] == "mlp":
            s["weights"] = dip.ExpertWeights(*(dip.GroupedMatrix(*s[n]) for n in ("gate", "up", "down")))
            s["buffers"] = dip.ExpertWork(c["tokens"], c["top_k"], s["weights"], "cuda")
            s["y"] = torch.empty((c["tokens"], c["d_model"]), device="cuda", dtype=torch.bfloat16)
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------------------
def _codes(v):
    """[n, d] binary32 -> e4m3 codes and [n, blocks] scales."""
    n, d = v.shape
    b = torch.nn.functional.pad(v, (0, -d % BLOCK)).view(n, -1, BLOCK)
    amax = b.abs().amax(dim=2)
    s = (amax / torch.full_like(amax, TOP)).clamp_min(TINY)              # (a quotient: torch multiplies by 1 / a number)
    return (b / s[:, :, None]).reshape(n, -1)[:, :d].to(torch.float8_e4m3fn), s


def _row_values(codes, scale):
    return codes.float() if scale is None else codes.float() * scale.repeat_interleave(BLOCK, dim=1)[:, :codes.shape[1]]


def _weight_values(w, scale):
    if scale is None:
        return w.float()
    blocks = scale.repeat_interleave(BLOCK, dim=1)[:, :w.shape[1]].repeat_interleave(BLOCK, dim=2)[:, :, :w.shape[2]]
    return w.float() * blocks


def _rounded(v, wtype):
    """What a product takes for v: 8-bit weights multiply 8-bit rows."""
    return _row_values(*_codes(v)) if wtype == "fp8" else v


def _choice(logits, top_k, renorm):
    """Each token's experts (-1: none is left) and weights."""
    z = logits.float()
    z = torch.where(torch.isnan(z), torch.full_like(z, -math.inf), z)
    expert = torch.argsort(z, dim=1, descending=True, stable=True)[:, :top_k]
    top = z.gather(1, expert)
    there = top > -math.inf
    high = z.amax(dim=1, keepdim=True)
    high = torch.where(there[:, :1], high, torch.zeros_like(high))
    part = torch.exp(top - high)
    whole = part.sum(dim=1, keepdim=True) if renorm else torch.exp(z - high).sum(dim=1, keepdim=True)
    weight = torch.where(there, part / whole, torch.zeros_like(part))
    return torch.where(there, expert, torch.full_like(expert, -1)), weight


def _groups(expert, experts):
    """The rows grouped by expert: each expert's first row, each row's token, each choice's row."""
    tokens, top_k = expert.shape
    key = torch.where(expert < 0, torch.full_like(expert, experts), expert).flatten()
    order = torch.argsort(key, stable=True)
    offset = torch.searchsorted(key[order], torch.arange(experts + 1, device=key.device))
    rank = torch.arange(tokens * top_k, device=key.device)
    row = torch.empty_like(order).scatter_(0, order, rank)
    row = torch.where(expert.flatten() < 0, torch.full_like(row, -1), row).view(tokens, top_k)
    row_token = torch.where(rank < offset[-1], order // top_k, torch.zeros_like(order))
    return offset.int(), row_token.int(), row.int()


def _grouped(values, row_expert, place, most, *matrices):
    """values[r] @ W[row_expert[r]].T for each matrix: few rows with a copy of their matrices, many in padded groups."""
    experts = matrices[0][0].shape[0]
    if values.shape[0] <= experts:
        return [torch.bmm(_weight_values(w[row_expert], s if s is None else s[row_expert]), values[:, :, None])[:, :, 0]
                for w, s in matrices]
    slot = row_expert * most + place
    padded = torch.zeros((experts * most, values.shape[1]), device=values.device).index_copy_(0, slot, values)
    padded = padded.view(experts, most, -1)
    return [torch.bmm(padded, _weight_values(w, s).transpose(1, 2)).view(experts * most, -1)[slot] for w, s in matrices]


def _silu(v):
    return v / (1 + torch.exp(-v))


def _plain(s):
    c = s["case"]
    if c["kind"] == "route":
        expert, weight = _choice(s["logits"], c["top_k"], c["renorm"])
        offset, row_token, row = _groups(expert, c["experts"])
        return {"expert": expert.int(), "weight": weight, "offset": offset, "row_token": row_token, "token_row": row}
    if c["kind"] == "product":
        e = s["row_expert"].long()
        place = torch.arange(c["rows"], device=e.device) - s["offset"].long()[e]
        return {"y": _grouped(_row_values(s["x"], s.get("x_scale")), e, place, s["most"], s["w"])[0].bfloat16()}
    x = _rounded(s["x"].float(), c["wtype"])
    if c["kind"] == "linear":
        return {"y": (x @ _weight_values(*s["w"])[0].t()).bfloat16()}
    if not c["top_k"]:
        gate, up, down = (_weight_values(*s[n])[0].t() for n in ("gate", "up", "down"))
        return {"y": (_rounded(_silu(x @ gate) * (x @ up), c["wtype"]) @ down).bfloat16()}
    expert, weight = _choice(s["logits"], c["top_k"], True)
    offset, row_token, row = _groups(expert, c["experts"])
    r = torch.arange(row_token.numel(), device=row.device)
    row_expert = torch.searchsorted(offset, r.int(), right=True) - 1
    place = r - offset.long()[row_expert]
    gate, up = _grouped(x[row_token.long()], row_expert, place, s["most"], s["gate"], s["up"])
    out = _grouped(_rounded(_silu(gate) * up, c["wtype"]), row_expert, place, s["most"], s["down"])[0]
    y = (out[row.long()] * weight[:, :, None]).sum(dim=1)
    return {"y": y.bfloat16(), "expert": expert.int(), "weight": weight}


# ---- one pass ----------------------------------------------------------------------------------------------------------
def _call(s):
    c, dip = s["case"], s["dip"]
    if c["kind"] == "route":
        r = s["route"]
        dip.dip_route_experts(_context, s["logits"], r, renormalize=c["renorm"])
        return {"expert": r.expert, "weight": r.weight, "offset": r.offset, "row_token": r.row_token, "token_row": r.token_row}
    if c["kind"] == "product":
        dip.dip_grouped_product(_context, s["matrix"], s["rows"], s["y"], offset=s["offset"])
        return {"y": s["y"]}
    if c["kind"] == "linear":
        if c["wtype"] == "fp8":
            dip.dip_stage_rows(_context, s["x"], s["rows"])
        dip.dip_grouped_product(_context, s["matrix"], s["rows"], s["y"])
        return {"y": s["y"]}
    if not c["top_k"]:
        dip.dip_expert_mlp(_context, s["weights"], s["x"], s["buffers"], s["y"])
        return {"y": s["y"]}
    r = s["route"]
    dip.dip_route_experts(_context, s["logits"], r)
    dip.dip_expert_mlp(_context, s["weights"], s["x"], s["buffers"], s["y"], route=r)
    return {"y": s["y"], "expert": r.expert, "weight": r.weight}


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
    if c["kind"] == "route":
        n = c["tokens"] * c["top_k"]
        return {"bytes": c["tokens"] * c["experts"] * (4.0 if c["logits"] == "f32" else 2.0) + 16.0 * n + 4.0 * (c["experts"] + 1),
                "flops": 4.0 * c["tokens"] * c["experts"]}
    item = 2.0 if c["wtype"] == "bf16" else 1.0 + 4.0 / BLOCK ** 2          # (a weight, with its share of the scales)
    if c["kind"] == "product":
        row = 2.0 * c["d_in"] if c["wtype"] == "bf16" else c["d_in"] * (1.0 + 4.0 / BLOCK)
        return {"bytes": _met(c["experts"], c["rows"]) * c["d_in"] * c["d_out"] * item + c["rows"] * (row + 2.0 * c["d_out"]),
                "flops": 2.0 * c["rows"] * c["d_in"] * c["d_out"]}
    if c["kind"] == "linear":
        return {"bytes": c["d_in"] * c["d_out"] * item + 2.0 * c["tokens"] * (c["d_in"] + c["d_out"]),
                "flops": 2.0 * c["tokens"] * c["d_in"] * c["d_out"]}
    rows = c["tokens"] * max(1, c["top_k"])
    met = c["experts"] * (1 - (1 - c["top_k"] / c["experts"]) ** c["tokens"]) if c["top_k"] else 1
    return {"bytes": met * 3 * c["d_model"] * c["d_ff"] * item + 4.0 * c["tokens"] * c["d_model"] + 4.0 * c["tokens"] * c["experts"],
            "flops": 6.0 * rows * c["d_model"] * c["d_ff"]}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------
def _quantised64(v):
    """The values that the 8-bit form of a row stands for; scale and quotient are binary32 numbers by definition."""
    out = torch.zeros_like(v)
    for b in range(0, v.shape[1], BLOCK):
        part = v[:, b:b + BLOCK]
        scale = torch.clamp_min((part.abs().amax(dim=1, keepdim=True).float().double() / TOP).float(), TINY).double()
        out[:, b:b + BLOCK] = (part / scale).float().to(torch.float8_e4m3fn).double() * scale
    return out


def _matrix64(w, scale, e):
    m = w[e].double()
    if scale is not None:
        for i in range(scale.shape[1]):
            for k in range(0, m.shape[1], BLOCK):
                m[i * BLOCK:(i + 1) * BLOCK, k:k + BLOCK] *= scale[e, i, k // BLOCK].double()
    return m


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    if "logits" in s:
        z = s["logits"].double()
        p = torch.softmax(z, dim=1).nan_to_num(0.0)
        weight, expert = torch.sort(p, dim=1, descending=True, stable=True)
        weight, expert = weight[:, :c["top_k"]].contiguous(), expert[:, :c["top_k"]]
        if c.get("renorm", True):
            weight = (weight / weight.sum(dim=1, keepdim=True)).nan_to_num(0.0)
        if c["kind"] == "route":
            return {"expert": None, "weight": weight, "offset": None, "row_token": None, "token_row": None}
    if c["kind"] == "product":
        y = torch.zeros((c["rows"], c["d_out"]), device="cuda", dtype=torch.float64)
        for e, (a, b) in enumerate(zip(s["offset"].tolist()[:-1], s["offset"].tolist()[1:])):
            if b > a:
                x = s["x"][a:b].double()
                if "x_scale" in s:
                    for k in range(0, c["d_in"], BLOCK):
                        x[:, k:k + BLOCK] *= s["x_scale"][a:b, k // BLOCK, None].double()
                y[a:b] = x @ _matrix64(*s["w"], e).t()
        return {"y": y}
    x = s["x"].double()
    if c["wtype"] == "fp8":
        x = _quantised64(x)
    if c["kind"] == "linear":
        return {"y": x @ _matrix64(*s["w"], 0).t()}
    y = torch.zeros((c["tokens"], c["d_model"]), device="cuda", dtype=torch.float64)
    for e in range(c["experts"]):
        at = torch.arange(c["tokens"], device="cuda") if not c["top_k"] else (expert == e).any(dim=1).nonzero()[:, 0]
        if not at.numel():
            continue
        gate, up = (x[at] @ _matrix64(*s[n], e).t() for n in ("gate", "up"))
        h = gate * torch.sigmoid(gate) * up
        out = (_quantised64(h) if c["wtype"] == "fp8" else h) @ _matrix64(*s["down"], e).t()
        share = (weight * (expert == e)).sum(dim=1, keepdim=True)[at] if c["top_k"] else 1.0
        y[at] += out * share
    return {"y": y} if not c["top_k"] else {"y": y, "expert": None, "weight": weight}
