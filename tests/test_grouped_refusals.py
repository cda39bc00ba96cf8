"""What the operators on groups and on gradients refuse, on the host: nothing is launched, so that no GPU is needed."""
import ctypes
import math

import pytest
import torch

import paper_2204_02662_amd as epp

BAD, LARGE = epp.EPP_ERR_INVALID_ARG, epp.EPP_ERR_TOO_LARGE
A = 1 << 20  # addresses that nobody reads


def rows(data=A, n=10, ld=16, list_=None):
    return ctypes.byref(epp._Rows(data, n, ld, list_))


@pytest.mark.parametrize("call", ["epp_grouped_product", "epp_grouped_input_gradient"])
def test_rows(call):
    lib = epp.load_library()
    fn = getattr(lib, call)

    def rc(type_=0, x=None, W=2 * A, offsets=3 * A, G=4, m=10, Fi=16, Fo=16, out=None):
        return fn(type_, rows() if x is None else x, W, offsets, G, m, Fi, Fo, rows(4 * A) if out is None else out, None)
    for want, bad in ((BAD, dict(type_=3)), (BAD, dict(type_=-1)), (BAD, dict(x=ctypes.POINTER(epp._Rows)())), (BAD, dict(W=None)),
                      (BAD, dict(offsets=None)), (BAD, dict(G=0)), (LARGE, dict(G=2049)), (BAD, dict(m=-1)), (LARGE, dict(m=1 << 31)),
                      (BAD, dict(Fi=0)), (BAD, dict(Fo=0)), (LARGE, dict(Fi=65_537)), (LARGE, dict(Fo=65_537)), (BAD, dict(m=11)),
                      (BAD, dict(x=rows(n=9))), (BAD, dict(x=rows(ld=15))), (BAD, dict(x=rows(data=None))), (BAD, dict(out=rows(4 * A, ld=15))),
                      (BAD, dict(out=rows(4 * A, n=9))), (BAD, dict(x=rows(n=-1))), (LARGE, dict(x=rows(n=1 << 31))), (BAD, dict(x=rows(A + 2))),
                      (BAD, dict(W=2 * A + 1)), (BAD, dict(offsets=3 * A + 2)), (BAD, dict(x=rows(list_=A + 1))),
                      # outputs on inputs' memory: the same matrix, its last element, columns that overlap, another distance of rows, W, offsets
                      (BAD, dict(out=rows(A))), (BAD, dict(out=rows(A + 4 * 159))), (BAD, dict(x=rows(ld=32), out=rows(A + 4 * 15, ld=32))),
                      (BAD, dict(x=rows(ld=32), out=rows(A + 4 * 17, ld=32))), (BAD, dict(x=rows(ld=32), out=rows(A + 4 * 16, ld=40))),
                      (BAD, dict(out=rows(2 * A + 4 * 1023))), (BAD, dict(out=rows(3 * A)))):
        assert rc(**bad) == want, bad
        assert lib.epp_last_error()
    # (different columns of one matrix, one row to a group or none: nothing to refuse, and with no entry nothing to launch)
    assert rc(m=0, x=rows(ld=32), out=rows(A + 4 * 16, ld=32)) == epp.EPP_OK
    assert rc(m=0, x=rows(data=None, n=0), out=rows(None, n=0)) == epp.EPP_OK


def test_weight_gradient():
    lib = epp.load_library()
    need = lib.epp_grouped_weight_gradient_workspace(10, 4, 16, 16)
    assert need > 0

    def rc(type_=1, x=None, d=None, offsets=3 * A, G=4, m=10, Fi=16, Fo=16, wtype=0, W=4 * A, ws=5 * A, bytes_=need):
        return lib.epp_grouped_weight_gradient(type_, x or rows(), rows(2 * A) if d is None else d, offsets, G, m, Fi, Fo, wtype, W, ws, bytes_, None)
    for want, bad in ((BAD, dict(type_=7)), (BAD, dict(wtype=2)), (BAD, dict(type_=0, wtype=1)), (BAD, dict(W=None)), (BAD, dict(ws=None)),
                      (BAD, dict(bytes_=need - 1)), (BAD, dict(ws=5 * A + 8)), (BAD, dict(G=0)), (LARGE, dict(G=2049)), (BAD, dict(m=11)),
                      (BAD, dict(d=rows(2 * A, ld=15))), (BAD, dict(offsets=None)), (BAD, dict(W=A)), (BAD, dict(W=2 * A + 16)),
                      (BAD, dict(W=4 * A + 2)), (BAD, dict(ws=4 * A)), (BAD, dict(ws=A))):
        assert rc(**bad) == want, bad
    for bad in ((-1, 4, 16, 16), (1 << 31, 4, 16, 16), (10, 0, 16, 16), (10, 2049, 16, 16), (10, 4, 0, 16), (10, 4, 16, 65_537)):
        assert lib.epp_grouped_weight_gradient_workspace(*bad) < 0
        with pytest.raises(epp.EppError):
            epp.epp_grouped_weight_gradient_workspace(*bad)


def test_grouped_launches_too_large():
    """More tiles of the result than a launch has workgroups for; offsets on memory that the weight gradient writes."""
    lib, m = epp.load_library(), (1 << 31) - 1
    B = 1 << 45

    def many(data, ld):
        return ctypes.byref(epp._Rows(data, m, ld, None))
    for type_, Fi, Fo in ((0, 128, 256), (1, 16, 16), (2, 24, 1000)):
        for fn in (lib.epp_grouped_product, lib.epp_grouped_input_gradient):
            assert fn(type_, many(A, 1024), A, A, 2048, m, Fi, Fo, many(B, 1024), None) == LARGE
            assert b"tiles" in lib.epp_last_error()
    assert lib.epp_grouped_weight_gradient(0, rows(ld=65_536), rows(2 * A, ld=65_536), A, 2048, 10, 65_536, 65_536, 0, B, B // 2, 16, None) == LARGE
    need = lib.epp_grouped_weight_gradient_workspace(10, 4, 16, 16)
    for offsets in (4 * A, 4 * A + 4 * 1020, 5 * A, 5 * A + need - 4):
        assert lib.epp_grouped_weight_gradient(1, rows(), rows(2 * A), offsets, 4, 10, 16, 16, 0, 4 * A, 5 * A, need, None) == BAD


def test_group_rows():
    lib = epp.load_library()
    need = lib.epp_group_rows_workspace(10_000, 8)
    assert need > 0

    def rc(group_of=A, n=20_000, rows_=2 * A, m=10_000, G=8, offsets=3 * A, order=4 * A, ws=5 * A, bytes_=need):
        return lib.epp_group_rows(group_of, n, rows_, m, G, offsets, order, ws, bytes_, None)
    for want, bad in ((BAD, dict(group_of=None)), (BAD, dict(rows_=None)), (BAD, dict(m=-1)), (LARGE, dict(m=1 << 31)), (BAD, dict(G=0)),
                      (LARGE, dict(G=2049)), (BAD, dict(offsets=None)), (BAD, dict(order=None)), (BAD, dict(ws=None)), (BAD, dict(bytes_=need - 4)),
                      (BAD, dict(ws=5 * A + 4)), (BAD, dict(n=-1)), (LARGE, dict(n=1 << 31)), (BAD, dict(group_of=A + 1)), (BAD, dict(order=A)),
                      (BAD, dict(order=2 * A + 39_996)), (BAD, dict(offsets=4 * A + 39_000)), (BAD, dict(ws=4 * A))):
        assert rc(**bad) == want, bad
    for bad in ((-1, 8), (1 << 31, 8), (5, 0), (5, 2049)):
        with pytest.raises(epp.EppError):
            epp.epp_group_rows_workspace(*bad)


def test_gradients():
    lib = epp.load_library()
    need = lib.epp_gradient_norm_workspace(2)
    assert need > 0 and lib.epp_gradient_norm_workspace(-1) == BAD and lib.epp_gradient_norm_workspace((1 << 20) + 1) == LARGE

    def table(*grads):
        return (epp._Gradient * len(grads))(*[epp._Gradient(*g) for g in grads])
    fine = [(A, None, 100, 0), (2 * A, None, 100, 1)]

    def clip(grads=fine, n=None, max_norm=1.0, norm=3 * A, ws=4 * A, bytes_=need):
        return lib.epp_clip_gradients(table(*grads) if grads is not None else None, len(grads) if n is None else n, max_norm, norm, ws, bytes_, None)
    for want, bad in ((BAD, dict(max_norm=-1.0)), (BAD, dict(max_norm=math.nan)), (BAD, dict(grads=None, n=2)), (BAD, dict(n=-1)),
                      (LARGE, dict(n=(1 << 20) + 1)), (BAD, dict(norm=None)), (BAD, dict(norm=3 * A + 2)), (BAD, dict(ws=None)), (BAD, dict(ws=4 * A + 8)),
                      (BAD, dict(bytes_=need - 8)), (BAD, dict(grads=[(None, None, 1, 0)])), (BAD, dict(grads=[(A, None, -1, 0)])),
                      (LARGE, dict(grads=[(A, None, 1 << 40, 0)])), (BAD, dict(grads=[(A, None, 5, 3)])), (BAD, dict(grads=[(A + 2, None, 5, 0)])),
                      (BAD, dict(grads=[(A, 2 * A + 1, 5, 1)])), (BAD, dict(grads=[fine[0], fine[0]])), (BAD, dict(grads=[fine[0], (A + 396, None, 1, 0)])),
                      (BAD, dict(grads=[(A, A + 4, 100, 0)])), (BAD, dict(grads=[(A, 2 * A, 100, 0), (2 * A, A, 100, 0)])), (BAD, dict(norm=A + 8)),
                      (BAD, dict(ws=A - need + 16)), (BAD, dict(norm=4 * A))):
        assert clip(**bad) == want, bad
    assert lib.epp_gradient_norm(table((A, None, 100, 0)), 1, A, 4 * A, need, None) == BAD


def test_tensors_that_are_not_on_the_gpu_or_of_another_kind():
    x, i = torch.zeros(4, 4), torch.zeros(5, dtype=torch.int32)
    b = torch.zeros(64, dtype=torch.uint8)
    for call in (lambda: epp.epp_group_rows(i, 4, i, i, b), lambda: epp.epp_grouped_product(x, x, i, x), lambda: epp.epp_grouped_input_gradient(x, x, i, x),
                 lambda: epp.epp_grouped_weight_gradient(x, x, i, x, b), lambda: epp.epp_gradient_norm([x], x, b), lambda: epp.epp_clip_gradients([x], 1.0, x, b)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: epp.epp_group_rows(i, 4, i), lambda: epp.epp_grouped_product(x, x, i, x, wrong=1), lambda: epp.epp_clip_gradients([x], 1.0),
                 lambda: epp.epp_grouped_product(1, x, i, x), lambda: epp.epp_gradient_norm([x], 3, b)):
        with pytest.raises(TypeError):
            call()
