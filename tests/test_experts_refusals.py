"""What the binding of the router and the grouped products refuses, before the library is called (no GPU needed)."""
import types

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture()
def dip(monkeypatch):
    import paper_2412_01380_b200 as dip

    class Reached(Exception):
        pass

    class Lib:
        def __getattr__(self, name):
            if name == "dip_status_string":
                return lambda st: b"invalid argument"
            raise Reached(name)

    monkeypatch.setattr(dip, "_lib", Lib())
    return dip


CTX = types.SimpleNamespace(device=0, handle=None)
BF16 = torch.bfloat16


def test_matrices(dip):
    for values, scales in [(torch.zeros(2, 64, 64), None), (torch.zeros((2, 64, 64), dtype=BF16), None),           # type; not on a device
                           (torch.zeros((2, 64, 64), dtype=torch.float16), None),
                           (torch.zeros((2, 64, 64), dtype=torch.uint8).view(torch.float8_e4m3fn), None)]:
        with pytest.raises(dip.DipError):
            dip.GroupedMatrix(values, scales)


@pytest.mark.parametrize("args", [(0, 8, 2), (65537, 8, 2), (4, 0, 1), (4, 513, 2), (4, 8, 9), (4, 8, 0), (4, 64, 17)])
def test_routes(dip, args):
    with pytest.raises(dip.DipError):
        dip.ExpertRoute(*args, "cpu")


def test_route_calls(dip):
    r = dip.ExpertRoute(4, 8, 2, "cpu")
    for logits in (torch.zeros(4, 8), torch.zeros((4, 8), dtype=torch.float64), None, torch.zeros(4, 7), torch.zeros(5, 8)):
        with pytest.raises(dip.DipError):
            dip.dip_route_experts(CTX, logits, r)


def test_rows_and_work(dip):
    with pytest.raises(dip.DipError):
        dip.Rows(4, 64, dip.W_F32, "cpu")
    with pytest.raises(dip.DipError):
        dip.Rows.of(torch.zeros((4, 64), dtype=BF16))
    rows = dip.Rows(4, 64, dip.W_BF16, "cpu")
    with pytest.raises(dip.DipError):
        dip.dip_stage_rows(CTX, torch.zeros((4, 64), dtype=BF16), rows)
    w = types.SimpleNamespace(wtype=dip.W_BF16, d_model=64, d_ff=96)
    for tokens, top_k in ((0, 2), (65537, 2), (4, 17), (4, -1)):
        with pytest.raises(dip.DipError):
            dip.ExpertWork(tokens, top_k, w, "cpu")


def test_null_arguments_of_the_library(dip):
    """The C entry points with nothing in their arguments: an error code, no crash."""
    import ctypes
    lib = ctypes.CDLL(dip.LIB_PATH)
    n = None
    for name, args in (("dip_route_experts", (n, n, 0, 0, n, n)), ("dip_stage_rows", (n, n, 1, 64, n, 1, n, n, n)),
                       ("dip_grouped_product", (n, n, n, n, 1, n, n, 0, n)), ("dip_grouped_gate_up", (n, n, n, n, n, 1, n, n, n, n)),
                       ("dip_combine_rows", (n, n, n, 64, n, n)), ("dip_expert_mlp", (n, n, n, n, n, 1, n, n, n, n))):
        assert getattr(lib, name)(*args) == dip.ERR_INVALID_ARG, name
