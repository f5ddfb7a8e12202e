"""What a context's options may not be, on the host alone (no GPU needed)."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")
import paper_2412_01380_b200 as dip


@pytest.mark.parametrize("name,values", [("max_d", (-1, 32769)), ("max_batch", (-1, 17)), ("gemv_segment_bytes", (1, 4096)),
                                         ("wait_limit_us", (-1,)), ("int4_kernel", (-1, 3))])
def test_options_outside_their_range(name, values):
    lib = C.CDLL(dip.LIB_PATH)
    for v in values:
        handle, opt = C.c_void_p(1), dip.OptionsStruct()
        setattr(opt, name, v)
        assert lib.dip_create_ex(C.byref(handle), 0, C.byref(opt)) == dip.ERR_INVALID_ARG
        assert not handle.value


def test_the_options_keep_their_size():
    """What was reserved becomes an option: programs that were compiled before pass zero there."""
    assert C.sizeof(dip.OptionsStruct) == 40 and dip.OptionsStruct.int4_kernel.offset == 28
