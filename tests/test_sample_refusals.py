"""What the choice of tokens refuses, on the host alone (no GPU needed): the binding, and the library's own checks with a device that only
says its number."""
import ctypes as C
import types

import pytest

torch = pytest.importorskip("torch")
import paper_2412_01380_b200 as dip

CTX = types.SimpleNamespace(device=0, handle=None)


def test_the_binding_refuses_before_the_library_is_called():
    z, u, t = torch.zeros((4, 10)), torch.zeros(4), torch.zeros(4, dtype=torch.int32)
    for args in ((z, u, t), (None, u, t), (z.half(), u, t)):
        with pytest.raises(dip.DipError):
            dip.dip_sample_tokens(CTX, *args)
    here = types.SimpleNamespace(device=-1, handle=None)           # (tensors without a device have -1)
    for args in ((z[0], u, t), (z.t(), u, t), (z[:0], u[:0], t[:0]), (z, u[:3], t), (z, u, t.long()), (z, None, t), (z, u, None)):
        with pytest.raises(dip.DipError):
            dip.dip_sample_tokens(here, *args)
    for name, value in (("top_k", u), ("top_p", t), ("temperature", u[:2]), ("min_p", u.double()), ("prob", t)):
        with pytest.raises(dip.DipError):
            dip.dip_sample_tokens(here, z, u, t, **{name: value})


def test_null_arguments():
    lib = C.CDLL(dip.LIB_PATH)
    assert lib.dip_sample_tokens(None, None, 0, 1, 10, C.c_int64(10), None, None, None, None, None) == dip.ERR_INVALID_ARG


def test_the_definition_by_hand():
    """The reference itself, on rows whose answers can be told without it."""
    import math

    import sample_util as su
    z = torch.tensor([0.0, math.log(2.0), math.log(4.0), math.log(2.0), -math.inf])          # 1, 2, 4, 2, closed: of 9
    assert su.choose(z, 0.0)[:2] == (0, pytest.approx(1 / 9))
    assert su.choose(z, 0.12)[0] == 1 and su.choose(z, 0.34)[0] == 2 and su.choose(z, 0.99)[0] == 3
    assert su.choose(z, 0.5, top_k=2)[:2] == (2, pytest.approx(4 / 6)) and su.choose(z, 0.1, top_k=2)[0] == 1     # 1 and 3 tie: the lower one
    assert su.choose(z, 0.99, top_p=0.4)[:2] == (2, 1.0)                                     # 4 of 9 reach 0.4
    assert su.choose(z, 0.99, top_p=0.45)[0] == 2 and su.choose(z, 0.1, top_p=0.45)[0] == 1  # 4 do not reach 0.45: one more
    assert su.choose(z, 0.99, top_k=3, top_p=0.5)[:2] == (2, 1.0)                            # 4 of 8 reach 0.5
    assert su.choose(z, 0.99, min_p=0.6)[:2] == (2, 1.0) and su.choose(z, 0.99, min_p=0.4)[0] == 3
    assert su.choose(z, 0.7, temperature=0.0)[:2] == (2, 1.0) and su.choose(torch.full((3,), -math.inf), 0.5)[:2] == (-1, 0.0)
