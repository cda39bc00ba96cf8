"""Which memory the products of rows that belong to groups may share, on the host: refused calls launch nothing, and accepted ones have no entry,
so that no GPU is needed."""
import ctypes

import pytest

import paper_2204_02662_amd as epp

BAD, OK = epp.EPP_ERR_INVALID_ARG, epp.EPP_OK
A = 1 << 20  # addresses that nobody reads


def rows(data, n=10, ld=16, list_=None):
    return ctypes.byref(epp._Rows(data, n, ld, list_))


@pytest.mark.parametrize("call", ["epp_grouped_product", "epp_grouped_input_gradient"])
def test_outputs_on_lists_of_rows(call):
    """10 entries; a result of 10 rows of 16 floats at 4 A, 640 bytes: a list of 40 bytes that begins or ends in it is refused."""
    fn = getattr(epp.load_library(), call)

    def rc(in_list=None, out_list=None, out_n=10):
        return fn(0, rows(A, list_=in_list), 2 * A, 3 * A, 4, 10, 16, 16, rows(4 * A, out_n, list_=out_list), None)
    for at in (4 * A, 4 * A + 636, 4 * A - 36, 4 * A + 100):
        assert rc(in_list=at) == BAD and b"alias" in epp.load_library().epp_last_error()
        assert rc(out_list=at) == BAD and b"alias" in epp.load_library().epp_last_error()
        assert rc(in_list=6 * A, out_list=at) == BAD


def test_weight_gradients_on_lists_of_rows():
    lib = epp.load_library()
    need = lib.epp_grouped_weight_gradient_workspace(10, 4, 16, 16)

    def rc(x_list=None, d_list=None):
        return lib.epp_grouped_weight_gradient(1, rows(A, list_=x_list), rows(2 * A, list_=d_list), 3 * A, 4, 10, 16, 16, 0, 4 * A, 5 * A, need, None)
    for at in (4 * A, 4 * A + 4096 - 4, 4 * A - 36, 5 * A, 5 * A + need - 4, 5 * A - 36):
        assert rc(x_list=at) == BAD and b"alias" in lib.epp_last_error()
        assert rc(d_list=at) == BAD and b"alias" in lib.epp_last_error()
        assert rc(x_list=6 * A, d_list=at) == BAD
