"""Plain 64-bit forms of the products with 4-bit weights, and how far a kernel may be from them.

Products (code - 8) * x are exact in binary32.  Sums of n of them, whatever their order and even if each addition truncates
(2^-23), are within n 2^-23 sum|w x| of the exact ones; each group's multiply-add by its scale and each addition of a part is one
rounding more: two per group are allowed.
"""
import math

import torch

import expert_util as eu

GROUP = 128


def groups_of(d):
    return -(-d // GROUP)


def matrix(gen, experts, d_out, d_in):
    """Codes over their whole range and scales of which neighbours differ by up to 16 times, so that a wrong one shows."""
    codes = torch.randint(0, 256, (experts, d_out, d_in // 2), generator=gen, device="cuda", dtype=torch.uint8)
    scales = torch.exp2(torch.rand((experts, groups_of(d_in), d_out), generator=gen, device="cuda") * 4 - 9).half()
    return codes, scales


def weights64(codes, scales, e):
    q = torch.stack((codes[e] & 15, codes[e] >> 4), dim=2).flatten(1).double() - 8
    return q * scales[e].double().t().repeat_interleave(GROUP, dim=1)[:, :q.shape[1]]


def product64(codes, scales, x, offset=None):
    """y and the bound on a binary32 sum's distance from it, [n_rows, d_out]; NaN where no expert has the row."""
    y = torch.full((x.shape[0], codes.shape[1]), math.nan, device="cuda", dtype=torch.float64)
    off = torch.zeros_like(y)
    k, x = x.shape[1], x.double()
    for e, a, b in eu.groups(offset, x.shape[0], codes.shape[0]):
        m = weights64(codes, scales, e)
        y[a:b] = x[a:b] @ m.t()
        off[a:b] = (x[a:b].abs() @ m.abs().t()) * (k + 2 * groups_of(k)) * 2.0 ** -23
    return y, off


def gated64(gate, up, x, offset=None):
    """h = silu(gate x) * (up x) and the bound on its distance in binary32."""
    g, dg = product64(*gate, x, offset)
    u, du = product64(*up, x, offset)
    silu = g * torch.sigmoid(g)
    # |silu'| <= 1.1; exp, quotient and product: a few units of the last place
    return silu * u, 1.1 * dg * u.abs() + silu.abs() * du + 1.1 * dg * du + 16 * 2.0 ** -23 * (silu * u).abs()
