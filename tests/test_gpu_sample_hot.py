"""The choice of tokens at temperatures beside which differences of logits vanish."""
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

import paper_2412_01380_b200 as dip

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = dip.Context(0)
    yield c
    assert c.device_status() == dip.DEVICE_OK
    c.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("temperature", [1e20, 1e38])
@pytest.mark.parametrize("top_p", [None, 0.9])
@pytest.mark.parametrize("near,far", [(3, 0), (50, 60), (1000, 400), (6000, 200), (30000, 20000)])
def test_a_min_p_of_one_keeps_the_largest_alone(ctx, near, far, top_p, temperature, dtype):
    """Weights of all others are below the largest one's, if by less than any binary64 number can tell: a min_p of 1 leaves the largest logit and its
    equals, however near the next ones are, and each of these is drawn alike.  (An infinite temperature makes all logits alike.)"""
    g = torch.Generator(device="cuda")
    g.manual_seed(near)
    n, vocab = 16, near + far + 2
    below = 4 * (1 - torch.finfo(dtype).eps)                       # a step or two below 4
    z = torch.full((n, vocab), below, device="cuda")
    z[:, near:] = torch.randn((n, far + 2), generator=g, device="cuda") * 0.5
    z = z[:, torch.randperm(vocab, generator=g, device="cuda")].contiguous()
    at = torch.randperm(vocab, generator=g, device="cuda")[:2].sort().values.tolist()
    z[:, at] = 4.0
    z = z.to(dtype)
    if top_p is not None:
        z[:, : at[0]] = -float("inf")                              # (what top_p keeps has the two in it: they come first)
    u = (torch.arange(n, device="cuda") + 0.5) / n
    how = dict(temperature=torch.full((n,), temperature, device="cuda"), min_p=torch.tensor([1.0, 2.0] * (n // 2), device="cuda"))
    if top_p is not None:
        how["top_p"] = torch.full((n,), top_p, device="cuda")
    token, prob = torch.full((n,), -7, device="cuda", dtype=torch.int32), torch.zeros((n,), device="cuda")
    dip.dip_sample_tokens(ctx, z, u, token, prob=prob, **how)
    assert token.tolist() == [at[0]] * (n // 2) + [at[1]] * (n // 2) and (prob == 0.5).all()
    how["temperature"].fill_(float("inf"))
    dip.dip_sample_tokens(ctx, z, u, token, prob=prob, **how)
    assert (prob < 0.5).all()
