"""The choice of tokens from rows that are apart: what lies between them is the caller's."""
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

import paper_2412_01380_b200 as dip
import sample_util as su

pytestmark = pytest.mark.gpu
N, VOCAB, PITCH = 4, 50, 64


@pytest.fixture(scope="module")
def ctx():
    c = dip.Context(0)
    yield c
    assert c.device_status() == dip.DEVICE_OK
    c.close()


def buffer(dtype):
    """The rows, and 32-bit views of the memory in which they lie (with a row's distance in front of them and behind them)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    memory = torch.randn(((N + 2) * PITCH,), generator=g, device="cuda").to(dtype)
    return memory[PITCH:-PITCH].view(N, PITCH)[:, :VOCAB], memory.view(torch.int32), memory.view(torch.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_tokens_and_probabilities_between_rows_in_front_and_behind(ctx, dtype):
    words = torch.finfo(dtype).bits / 32                           # 32-bit words per item
    start, each, apart = int(PITCH * words), int(VOCAB * words), int(PITCH * words)
    u = torch.tensor([0.1, 0.5, 0.8, 0.99], device="cuda")
    last = start + (N - 1) * apart
    for at in (start - N, last + each, *(start + r * apart + each for r in range(N - 1)), *(start + (r + 1) * apart - N for r in range(N - 1))):
        for prob_too in (False, True):
            z, ints, floats = buffer(dtype)
            before, rows = ints.clone(), z.cpu()
            if prob_too:
                token, prob, got = torch.zeros((N,), device="cuda", dtype=torch.int32), floats[at:at + N], floats
            else:
                token, prob, got = ints[at:at + N], None, ints
            dip.dip_sample_tokens(ctx, z, u, token, prob=prob)
            want = [su.choose(rows[r], float(u[r])) for r in range(N)]
            assert token.tolist() == [w[0] for w in want]
            if prob_too:
                assert all(abs(p - w[1]) <= w[1] * (2.0 ** -24 + 2.0 ** -27) for p, w in zip(prob.tolist(), want))
            changed = torch.nonzero(got.view(torch.int32) != before).flatten().tolist()
            assert all(at <= i < at + N for i in changed)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_not_over_the_rows(ctx, dtype):
    words = torch.finfo(dtype).bits / 32
    start, each, apart = int(PITCH * words), int(VOCAB * words), int(PITCH * words)
    z, ints, floats = buffer(dtype)
    before, u = ints.clone(), torch.rand((N,), device="cuda")
    token = torch.full((N,), 9, device="cuda", dtype=torch.int32)
    for r in range(N):
        row = start + r * apart
        for at in (row - N + 1, row - 1, row, row + each // 2, row + each - 1):
            for args, kw in (((z, u, ints[at:at + N]), {}), ((z, u, token), dict(prob=floats[at:at + N]))):
                with pytest.raises(dip.DipError) as e:
                    dip.dip_sample_tokens(ctx, *args, **kw)
                assert e.value.status == dip.ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert torch.equal(ints, before) and (token == 9).all()
