"""Plain 64-bit forms of the router, the grouped products and the expert block, and how far a kernel may be from them.

Half a step of a rounding, relative to the value: bf16 2^-8, e4m3 2^-4 (2^-10 of the scale among its subnormals), binary32 2^-24.
Sums of n products in binary32, whatever their order and even if each addition truncates (2^-23), are within
n 2^-23 sum|a b| of the exact ones; a block's scale product and its multiply-add are two more roundings per block.
"""
import math

import torch

BLOCK = 128
TINY = 2.0 ** -126
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def blocks(d):
    return -(-d // BLOCK)


def quantise(v):
    """[n, d] of any float type -> codes, scales; scale and quotient are binary32 numbers."""
    n, d = v.shape
    b = torch.nn.functional.pad(v.float(), (0, -d % BLOCK)).view(n, -1, BLOCK)
    amax = b.abs().amax(dim=2)
    s = (amax / torch.full_like(amax, 448.0)).clamp_min(TINY)
    q = (b / s[:, :, None]).reshape(n, -1)[:, :d]
    return q.to(torch.float8_e4m3fn), s


def matrix(gen, fp8, experts, d_out, d_in, scale=0.05):
    """Weights and scales; the scales of neighbouring blocks differ by up to 16 times, so that a wrong one shows."""
    z = torch.randn((experts, d_out, d_in), generator=gen, device="cuda") * scale
    if not fp8:
        return z.bfloat16(), None
    s = torch.exp2(torch.rand((experts, blocks(d_out), blocks(d_in)), generator=gen, device="cuda") * 4 - 12)
    return (z / 2.0 ** -9).clamp(-448, 448).to(torch.float8_e4m3fn), s


def rows_of(gen, fp8, n, d):
    x = torch.randn((n, d), generator=gen, device="cuda").bfloat16()
    if not fp8:
        return x, None
    q, s = quantise(x * torch.exp2(torch.randint(-3, 4, (n, 1), generator=gen, device="cuda").float()).bfloat16())
    return q, s


def values64(q, s):
    v = q.double()
    return v if s is None else v * s.double().repeat_interleave(BLOCK, dim=-1)[..., :v.shape[-1]]


def weights64(w, s, e):
    v = w[e].double()
    if s is None:
        return v
    b = s[e].double().repeat_interleave(BLOCK, dim=0)[:v.shape[0]].repeat_interleave(BLOCK, dim=1)[:, :v.shape[1]]
    return v * b


def groups(offset, n_rows, experts):
    if offset is None:
        return [(0, 0, n_rows)]
    found, last = [], 0
    for e, (a, b) in enumerate(zip(offset.tolist()[:-1], offset.tolist()[1:])):
        a, b = max(last, min(a, n_rows)), min(b, n_rows)           # an offset below one in front of it counts as that one
        last = max(a, b)
        if b > a:
            found.append((e, a, b))
    return found


def product64(w, s, x, offset=None):
    """y and the bound on a binary32 sum's distance from it, [n_rows, d_out]; NaN where no expert has the row."""
    y = torch.full((x.shape[0], w.shape[1]), math.nan, device="cuda", dtype=torch.float64)
    off = torch.zeros_like(y)
    k = x.shape[1]
    for e, a, b in groups(offset, x.shape[0], w.shape[0]):
        m = weights64(w, s, e)
        y[a:b] = x[a:b] @ m.t()
        off[a:b] = (x[a:b].abs() @ m.abs().t()) * (k + 2 * blocks(k)) * 2.0 ** -23
    return y, off


def gated64(gate, up, x, offset=None):
    """h = silu(gate x) * (up x) and the bound on its distance in binary32."""
    g, dg = product64(*gate, x, offset)
    u, du = product64(*up, x, offset)
    silu = g * torch.sigmoid(g)
    h = silu * u
    # |silu'| <= 1.1; exp, quotient and product: a few units of the last place
    return h, 1.1 * dg * u.abs() + silu.abs() * du + 1.1 * dg * du + 16 * 2.0 ** -23 * h.abs()


def assert_within(got, want, bound, what=""):
    got, want = got.double(), want.double()
    bad = ~((got - want).abs() <= bound)
    if bad.any():
        i = tuple(torch.nonzero(bad)[0].tolist())
        raise AssertionError("%s: %d of %d values are too far off, the first at %s: %g for %g, %g allowed" % (
            what, int(bad.sum()), bad.numel(), i, got[i], want[i], bound[i] if torch.is_tensor(bound) else bound))


def rounded(want, bound, dtype):
    """The bound after one rounding to dtype."""
    return bound + HALF[dtype] * (want.abs() + bound)


def route64(logits, top_k, renormalize):
    """experts, weights, offsets, row_token, token_row, one token after the other."""
    z = logits.double().cpu()
    tokens, experts = z.shape
    expert = torch.full((tokens, top_k), -1, dtype=torch.int32)
    weight = torch.zeros((tokens, top_k), dtype=torch.float64)
    for t in range(tokens):
        row = z[t].tolist()
        open_ = [e for e in range(experts) if row[e] > -math.inf]        # (false for NaN)
        if not open_:
            continue
        high = max(row[e] for e in open_)
        part = {e: (1.0 if row[e] == math.inf else 0.0) if high == math.inf else math.exp(row[e] - high) for e in open_}
        best = sorted(open_, key=lambda e: (-row[e], e))[:top_k]
        total = sum(part[e] for e in (best if renormalize else open_))
        for j, e in enumerate(best):
            expert[t, j], weight[t, j] = e, part[e] / total
    order = [(int(expert[t, j]), t, j) for t in range(tokens) for j in range(top_k) if expert[t, j] >= 0]
    order.sort()
    token_row = torch.full((tokens, top_k), -1, dtype=torch.int32)
    for r, (_, t, j) in enumerate(order):
        token_row[t, j] = r
    offset = [sum(e < i for e, _, _ in order) for i in range(experts + 1)] if tokens * experts < 5000 else \
        torch.searchsorted(torch.tensor([e for e, _, _ in order]), torch.arange(experts + 1)).tolist()
    return expert, weight, torch.tensor(offset, dtype=torch.int32), torch.tensor([t for _, t, _ in order], dtype=torch.int32), token_row


def offsets(counts):
    o = [0]
    for c in counts:
        o.append(o[-1] + c)
    return torch.tensor(o, dtype=torch.int32, device="cuda")
