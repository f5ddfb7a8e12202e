"""What the binding keeps when the library refuses a call of the router or the products (no GPU needed)."""
import types

import pytest

torch = pytest.importorskip("torch")
import paper_2412_01380_b200 as dip


class Refuses:
    """A library whose calls all return DIP_ERR_INVALID_ARG."""

    def __getattr__(self, name):
        if name == "dip_status_string":
            return lambda status: b"invalid argument"
        if name == "dip_last_error":
            return lambda handle: b""
        return lambda *args: dip.ERR_INVALID_ARG


def context():
    c = types.SimpleNamespace(device=-1, handle=None)            # (tensors without a device have -1)
    c.check = lambda status: dip.Context.check(c, status)
    return c


@pytest.fixture()
def refusing(monkeypatch):
    monkeypatch.setattr(dip, "_lib", Refuses())
    monkeypatch.setattr(dip, "_stream", lambda: None)


def test_a_refused_router_call_leaves_the_route_as_it_was(refusing):
    route = dip.ExpertRoute(9, 8, 2, "cpu")
    route.struct.n_tokens = 9                                    # a call before
    with pytest.raises(dip.DipError):
        dip.dip_route_experts(context(), torch.zeros((4, 8)), route)
    assert route.n_tokens == 9 and route.n_rows == 18


def test_refused_calls_leave_the_rows_in_use_as_they_were(refusing):
    rows, h = dip.Rows(9, 64, dip.W_BF16, "cpu"), dip.Rows(9, 96, dip.W_BF16, "cpu")
    rows.n_rows, h.n_rows = 5, 7
    with pytest.raises(dip.DipError):
        dip.dip_stage_rows(context(), torch.zeros((9, 64), dtype=torch.bfloat16), rows)
    gate = types.SimpleNamespace(device=-1, wtype=dip.W_BF16, d_in=64, d_out=96, n_experts=1, ref=None)
    with pytest.raises(dip.DipError):
        dip.dip_grouped_gate_up(context(), gate, gate, rows, h)
    assert rows.n_rows == 5 and h.n_rows == 7
