"""The router's other forms against a 64-bit form: more than 4096 tokens (four to a warp, blocks of 128), more than 16384 (the counts
are added up by a launch of their own), more than 128 experts (choices without a sort), bfloat16 logits that share a word with their
index: experts, grouping and weights, over all experts and over the chosen ones."""
import math

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

import paper_2412_01380_b200 as dip
import expert_util as eu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = dip.Context(0)
    yield c
    assert c.device_status() == dip.DEVICE_OK
    c.close()


def form64(logits, top_k, renormalize):
    """expert, weight [tokens, top_k], offset, row_token, token_row."""
    z = logits.double() + 0.0                                      # (-0 is 0)
    tokens, experts = z.shape
    z = torch.where(torch.isnan(z), -math.inf, z)
    expert = torch.argsort(z, dim=1, descending=True, stable=True)[:, :top_k]
    top = z.gather(1, expert)
    there = top > -math.inf
    high = z.amax(dim=1, keepdim=True)
    # where +infinity stands, it shares the sum evenly
    part = torch.where(high == math.inf, (z == math.inf).double(), torch.exp(z - torch.where(high.isfinite(), high, 0.0)))
    chosen = part.gather(1, expert)
    total = (chosen if renormalize else part).sum(dim=1, keepdim=True)
    weight = torch.where(there, chosen / total, 0.0)
    expert = torch.where(there, expert, -1)
    key = torch.where(expert < 0, experts, expert).flatten()
    order = torch.argsort(key, stable=True)
    offset = torch.searchsorted(key[order], torch.arange(experts + 1, device=key.device)).int()
    row = torch.empty_like(order).scatter_(0, order, torch.arange(order.numel(), device=order.device))
    return expert.int(), weight, offset, (order // top_k)[:int(offset[-1])].int(), torch.where(key == experts, -1, row).view(tokens, top_k).int()


def logits_of(tokens, experts, dtype, seed):
    """Many ties (eighths), closed experts, NaN, padding, tokens with less than top_k open experts, +infinity."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    z = torch.randn((tokens, experts), generator=g, device="cuda") * 2
    ties = torch.arange(tokens, device="cuda") % 2 == 0
    z[ties] = (z[ties] * 8).round() / 8
    draw = torch.rand(z.shape, generator=g, device="cuda")
    z[draw < 0.3] = -math.inf
    z[draw > 0.99] = math.nan
    z[::7] = -math.inf
    z[2::101] = -math.inf
    z[2::101, experts - 1] = -3.0
    z[3::97, experts // 2] = math.inf
    z[3::97, 0] = math.inf
    z[4::89] = torch.finfo(torch.bfloat16).min                     # the lowest finite value: open, and all alike
    return z.bfloat16() if dtype == "bf16" else z


@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,experts,top_k", [
    (5, 200, 8), (31, 512, 16), (33, 512, 16), (128, 129, 4), (1000, 257, 5),
    (4096, 64, 8), (4097, 20, 3), (4097, 60, 6), (4097, 100, 16), (4100, 256, 8), (4223, 512, 16),
    (16384, 128, 8), (16384, 200, 8), (16385, 33, 6), (16385, 300, 4), (20001, 256, 2),
])
def test_route(ctx, tokens, experts, top_k, dtype, renormalize):
    z = logits_of(tokens, experts, dtype, tokens + experts)
    r = dip.ExpertRoute(tokens, experts, top_k, "cuda")
    r.row_token.fill_(-7)
    r.weight.fill_(math.nan)
    dip.dip_route_experts(ctx, z, r, renormalize=renormalize)
    expert, weight, offset, row_token, token_row = form64(z, top_k, renormalize)
    assert torch.equal(r.expert, expert)
    assert torch.equal(r.offset, offset)
    assert torch.equal(r.token_row, token_row)
    n = int(offset[-1])
    assert torch.equal(r.row_token[:n], row_token) and (r.row_token[n:] == -7).all()
    # exp(v - max) in binary32: the difference of two values of at most `big` is rounded by 2^-24 of twice that (values as far apart as the
    # lowest finite ones have exp = 0 on both sides), exp to 2 units of 2^-23, sums of up to `experts` parts, a quotient
    ordinary = z.float()[torch.isfinite(z) & (z > -1e30)]
    big = ordinary.abs().max().item()
    eu.assert_within(r.weight, weight, weight * ((4 * big + experts + 16) * 2.0 ** -24) + 2.0 ** -126, "weight")
