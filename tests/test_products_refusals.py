"""Calls that the products by list and the 8-bit products refuse, on the host: nothing here reaches a device.  (Pointers are
numbers that nobody follows.)"""
import ctypes as C

import pytest
import torch

from paper_2602_23999_amd import rabitq

P = 1 << 20  # an address, aligned


def _ls(groups=4, nprobe=2, pairs=6, n=8, k=16, off=P, ids=P):
    return rabitq._Lists(groups, nprobe, pairs, n, k, off, ids)


def _calls():
    lib = rabitq.load_library()

    def fwd(ls=None, dtype=2, x=P, ldx=16, w=P, ldw=16, stride=128, out=P, ldo=8):
        return lib.rabitq_grouped_matmul(C.byref(ls or _ls()), dtype, x, ldx, w, ldw, stride, out, ldo, None)

    def dx(ls=None, dtype=2, dout=P, ldd=8, w=P, ldw=16, stride=128, out=P, ldo=16, scratch=P):
        return lib.rabitq_grouped_matmul_dx(C.byref(ls or _ls()), dtype, dout, ldd, w, ldw, stride, out, ldo, scratch, None)

    def dw(ls=None, dtype=2, dout=P, ldd=8, x=P, ldx=16, out=P, ldo=16, stride=128):
        return lib.rabitq_grouped_matmul_dw(C.byref(ls or _ls()), dtype, dout, ldd, x, ldx, out, ldo, stride, P, None)

    def gi8(ls=None, x=P, ldx=16, sx=P, w=P, ldw=16, stride=128, sw=P, out=P, dtype=0, ldo=8):
        return lib.rabitq_grouped_matmul_i8(C.byref(ls or _ls()), x, ldx, sx, w, ldw, stride, sw, out, dtype, ldo, None)

    def i8(a=P, lda=16, sa=P, b=P, ldb=16, sb=P, m=3, n=5, k=16, out=P, dtype=0, ldo=5):
        return lib.rabitq_matmul_i8(a, lda, sa, b, ldb, sb, m, n, k, out, dtype, ldo, None)

    def quant(x=P, dtype=2, ldx=16, rows=3, k=16, codes=P, ldc=16, scale=P):
        return lib.rabitq_quantize_rows(x, dtype, ldx, rows, k, codes, ldc, scale, None)
    return dict(fwd=fwd, dx=dx, dw=dw, gi8=gi8, i8=i8, quant=quant)


BAD_LISTS = [dict(groups=0), dict(groups=-1), dict(nprobe=0), dict(pairs=-2), dict(pairs=7), dict(pairs=1 << 31),
             dict(n=0), dict(k=0), dict(n=(1 << 20) + 1), dict(k=(1 << 20) + 1), dict(off=None), dict(off=P + 2),
             dict(ids=P + 1)]


@pytest.mark.parametrize("name", ["fwd", "dx", "dw", "gi8"])
@pytest.mark.parametrize("bad", BAD_LISTS, ids=str)
def test_lists_out_of_range(name, bad):
    assert _calls()[name](ls=_ls(**bad)) == -1
    assert rabitq.load_library().rabitq_last_error()


@pytest.mark.parametrize("name,bad", [
    ("fwd", dict(dtype=3)), ("fwd", dict(dtype=-1)), ("fwd", dict(x=None)), ("fwd", dict(w=None)), ("fwd", dict(out=None)),
    ("fwd", dict(ldx=15)), ("fwd", dict(ldw=15)), ("fwd", dict(ldo=7)), ("fwd", dict(stride=127)), ("fwd", dict(stride=0)),
    ("fwd", dict(x=P + 1)), ("fwd", dict(out=P + 1)), ("fwd", dict(w=P + 2, dtype=0)),
    ("dx", dict(dtype=9)), ("dx", dict(dout=None)), ("dx", dict(w=None)), ("dx", dict(out=None)), ("dx", dict(scratch=None)),
    ("dx", dict(scratch=P + 8)), ("dx", dict(ldd=7)), ("dx", dict(ldw=15)), ("dx", dict(ldo=15)), ("dx", dict(stride=100)),
    ("dw", dict(dtype=4)), ("dw", dict(dout=None)), ("dw", dict(x=None)), ("dw", dict(out=None)), ("dw", dict(ldd=7)),
    ("dw", dict(ldx=15)), ("dw", dict(ldo=15)), ("dw", dict(stride=127)), ("dw", dict(dout=P + 1)),
    ("gi8", dict(dtype=3)), ("gi8", dict(x=None)), ("gi8", dict(w=None)), ("gi8", dict(sx=None)), ("gi8", dict(sw=None)),
    ("gi8", dict(out=None)), ("gi8", dict(ldx=15)), ("gi8", dict(ldw=15)), ("gi8", dict(ldo=7)), ("gi8", dict(stride=5)),
    ("gi8", dict(sx=P + 2)),
    ("i8", dict(dtype=3)), ("i8", dict(m=-1)), ("i8", dict(n=-1)), ("i8", dict(k=0)), ("i8", dict(k=131072, lda=131072, ldb=131072)),
    ("i8", dict(lda=15)), ("i8", dict(ldb=15)), ("i8", dict(ldo=4)), ("i8", dict(a=None)), ("i8", dict(b=None)),
    ("i8", dict(sa=None)), ("i8", dict(sb=None)), ("i8", dict(out=None)), ("i8", dict(m=1 << 31)), ("i8", dict(out=P + 2)),
    ("quant", dict(dtype=3)), ("quant", dict(rows=-1)), ("quant", dict(k=0)), ("quant", dict(k=(1 << 20) + 1, ldx=1 << 21, ldc=1 << 21)),
    ("quant", dict(ldx=15)), ("quant", dict(ldc=15)), ("quant", dict(x=None)), ("quant", dict(codes=None)),
    ("quant", dict(scale=None)), ("quant", dict(x=P + 1)), ("quant", dict(scale=P + 2)),
], ids=str)
def test_arguments_out_of_range(name, bad):
    assert _calls()[name](**bad) == -1
    assert rabitq.load_library().rabitq_last_error()


@pytest.mark.parametrize("name", ["fwd", "dx", "dw", "gi8"])
def test_number_of_lists_is_bounded(name):
    assert _calls()[name](ls=_ls(groups=(1 << 24) + 1)) == -1
    assert b"2^24" in rabitq.load_library().rabitq_last_error()


def test_sizes_behind_32_bits_are_not_cut_off():
    big = (1 << 32) + 16
    off = torch.zeros(5, dtype=torch.int32)
    for sizes in ((big, 8, 16), (4, big, 16), (4, 8, big)):
        with pytest.raises(rabitq.RabitqError, match="too many"):
            rabitq._lists_of(*sizes, 6, 2, off, None, 0)


def test_k_of_codes_by_list_is_bounded():
    k = 131072
    assert _calls()["gi8"](ls=_ls(k=k), ldx=k, ldw=k, stride=8 * k) == -1
    assert b"131071" in rabitq.load_library().rabitq_last_error()


def test_more_work_than_a_launch_holds():
    big = (1 << 31) - 1
    c = _calls()
    assert c["i8"](m=big, n=big, ldo=big) == -1
    assert b"too many tiles" in rabitq.load_library().rabitq_last_error()
    ls = dict(pairs=big - 1, n=1 << 20, k=16)
    assert c["fwd"](ls=_ls(**ls), ldo=1 << 20, stride=1 << 24) == -1
    assert c["dx"](ls=_ls(pairs=big - 1, k=1 << 20), ldw=1 << 20, ldo=1 << 20, stride=1 << 23) == -1
    wide = 1 << 20
    assert c["dw"](ls=_ls(groups=64, n=wide, k=wide), ldd=wide, ldx=wide, ldo=wide, stride=1 << 40) == -1
    assert c["quant"](rows=1 << 40, k=8192, ldx=8192, ldc=8192) == -1
    assert b"too many rows" in rabitq.load_library().rabitq_last_error()


def test_null_lists():
    lib = rabitq.load_library()
    assert lib.rabitq_grouped_matmul(None, 0, P, 16, P, 16, 128, P, 8, None) == -1
    assert lib.rabitq_grouped_dx_scratch_bytes(None) == -1 and lib.rabitq_grouped_dw_scratch_bytes(None) == -1


def test_nothing_to_do_needs_no_device():
    c = _calls()
    assert c["fwd"](ls=_ls(pairs=0), x=None, w=None, out=None) == 0
    assert c["dx"](ls=_ls(pairs=0), dout=None, w=None, out=None, scratch=None) == 0
    assert c["gi8"](ls=_ls(pairs=0), x=None, w=None, out=None, sx=None, sw=None) == 0
    assert c["i8"](m=0, a=None, sa=None, out=None) == 0 and c["i8"](n=0, b=None, sb=None, out=None, ldo=0) == 0
    assert c["quant"](rows=0, x=None, codes=None, scale=None) == 0


def test_scratch_sizes():
    lib = rabitq.load_library()
    assert lib.rabitq_grouped_dx_scratch_bytes(C.byref(_ls(nprobe=1))) == 0
    assert lib.rabitq_grouped_dx_scratch_bytes(C.byref(_ls())) >= 6 * 16 * 4 + 6
    assert lib.rabitq_grouped_dx_scratch_bytes(C.byref(_ls(groups=0))) == -1
    assert lib.rabitq_grouped_dw_scratch_bytes(C.byref(_ls())) >= 0


def test_binding_structure_matches_the_header():
    from test_abi import _header_structs
    assert [f[0] for f in rabitq._Lists._fields_] == _header_structs()["rabitq_lists"]


def test_binding_takes_tensors_of_the_device_only():
    x, w = torch.zeros(2, 4), torch.zeros(3, 5, 4)
    off = torch.zeros(4, dtype=torch.int32)
    for call in (lambda: rabitq.grouped_matmul(x, w, off), lambda: rabitq.grouped_matmul_dx(torch.zeros(2, 5), w, off),
                 lambda: rabitq.grouped_matmul_dw(torch.zeros(2, 5), x, off), lambda: rabitq.quantize_rows(x),
                 lambda: rabitq.matmul_i8(x.to(torch.int8), torch.ones(2), x.to(torch.int8), torch.ones(2)),
                 lambda: rabitq.grouped_matmul_i8(x.to(torch.int8), torch.ones(2), w.to(torch.int8), torch.ones(3, 5), off)):
        with pytest.raises(rabitq.RabitqError, match="current CUDA device"):
            call()
    for bad in (x.double(), x.int(), None):
        with pytest.raises(rabitq.RabitqError):
            rabitq.grouped_matmul(bad, w, off)
