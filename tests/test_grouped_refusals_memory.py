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


@pytest.mark.parametrize("call", ["epp_grouped_product", "epp_grouped_input_gradient"])
def test_columns_of_one_wider_matrix(call):
    """10 rows of 32 floats at A: inputs in the first 16 columns, outputs in the last 16, all rows, one of them or every second one."""
    fn = getattr(epp.load_library(), call)

    def rc(x, out):
        return fn(0, x, 2 * A, 3 * A, 4, 0, 16, 16, out, None)
    row = 4 * 32
    for first, second in ((A, A + 64), (A + 64, A)):  # columns of the one and of the other
        for step in (1, 2, 3):
            for other in (1, 2, 3):
                assert rc(rows(first, n=10 // step, ld=32 * step), rows(second, n=10 // other, ld=32 * other)) == OK
        for at in (0, 3, 9):
            # (a single row may have any distance from row to row)
            for ld in (16, 32, 1000):
                assert rc(rows(first + at * row, n=1, ld=ld), rows(second, ld=32)) == OK
                assert rc(rows(first, ld=32), rows(second + at * row, n=1, ld=ld)) == OK
    # a column too many, to either side; the same columns; single rows that share an element
    for at in (0, 3, 9):
        for off in (60, -60, 0, 4):
            if at * row + off < 0 or (off > 0 and at == 9):
                continue
            for ld in (16, 32):
                assert rc(rows(A + at * row + off, n=1, ld=ld), rows(A, ld=32)) == BAD
                assert rc(rows(A, ld=32), rows(A + at * row + off, n=1, ld=ld)) == BAD
        assert rc(rows(A + at * row, n=1), rows(A + at * row + 60, n=1)) == BAD
    assert rc(rows(A, n=5, ld=64), rows(A + 60, ld=32)) == BAD
    assert rc(rows(A, n=5, ld=64), rows(A + 68, ld=32)) == BAD
    assert rc(rows(A, n=3, ld=48), rows(A + 64, ld=32)) == BAD  # (its second row lies in the other's last columns)
    # a single row wider than the distance of the other's rows
    F_in, F_out = (64, 16) if call == "epp_grouped_product" else (16, 64)
    assert fn(0, rows(A, n=1, ld=64), 2 * A, 3 * A, 4, 0, F_in, F_out, rows(A + 64, n=3, ld=32), None) == BAD
