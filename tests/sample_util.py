"""The choice of a token, one row at a time in 64 bits, straight from its definition (CPU tensors)."""
import math

import torch


def choose(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """token, probability, and how near the number drawn is to a neighbouring token's range (as a share of the whole)."""
    z = z.double()
    z = torch.where(torch.isnan(z), torch.full_like(z, -math.inf), z)
    high = z.max()
    if high == -math.inf:
        return -1, 0.0, 1.0
    order = torch.sort(z, descending=True, stable=True).indices
    if not temperature > 0:
        return int(order[0]), 1.0, 1.0
    if high == math.inf:
        e = (z == math.inf).double()
    else:
        e = torch.exp((z - high) / temperature)
        e[z == -math.inf] = 0.0
        e[z == high] = 1.0
    order = order[z[order] > -math.inf]
    if 0 < top_k < z.numel():
        order = order[:top_k]
    if top_p < 1:
        mass = e[order].cumsum(0)
        before = torch.cat((torch.zeros(1, dtype=torch.float64), mass[:-1]))
        keep = before < max(top_p, 0.0) * mass[-1]
        keep[0] = True
        order = order[keep]
    if min_p > 0:
        order = order[e[order] >= min(min_p, 1.0)]
    kept = torch.zeros_like(e)
    kept[order] = e[order]
    cum = kept.cumsum(0)
    u = 0.0 if math.isnan(u) else min(max(u, 0.0), 1.0)
    at = u * float(cum[-1])
    above = torch.nonzero(cum > at)
    token = int(above[0]) if above.numel() else int(torch.nonzero(kept > 0)[-1])
    edge = float(min((cum[token] - at).abs(), (at - (cum[token] - kept[token])).abs()) / cum[-1])
    return token, float(kept[token] / cum[-1]), edge
