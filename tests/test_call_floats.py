"""What a record of a call holds of a Python float: its 32 bits where the function takes a float, the whole number it stands for elsewhere, as a
record of any other number."""
import ctypes as C
import struct

import pytest

torch = pytest.importorskip("torch")

from paper_1805_07941_amd import binding as B

A = [(i + 1) << 32 for i in range(8)]


def words(fn, args):
    n = len(args)
    return B.CallList([(fn, args)])._records.tolist()[1:1 + n]


def test_a_float_where_a_whole_number_belongs():
    L = B.lib()
    args = (A[0], 63.0, 1, 3.0, 64.0, A[1], 64, A[2], 4, 1, 0.0)
    assert words(L.dfq_quantize_mx, args) == [int(a) for a in args]
    args = (A[0], A[1], 8.0, B.fmt(4))
    assert words(L.dfq_quantize, args) == [A[0], A[1], 8, 4]
    with pytest.raises(B.DfqError) as e:                      # rows of 63 for K = 64: a size that says what it is
        B.CallList([(L.dfq_quantize_mx, (A[0], 63.0, 1, 3.0, 64.0, A[1], 64, A[2], 4, 1, 0))]).run(None)
    assert e.value.status == B.ESHAPE


def test_what_a_float_argument_is_given():
    fn = B.lib().dfq_rms_norm_mx
    args = [A[0], 63.0, None, 0, None, 0, 1, None, 1, 0, A[4], 64, None, 0, None, 0, 1, 0, 3, 64]
    for eps in (1e-6, 0, 1, 0.5, float("inf"), 1e39, 1e-50, 0x7f800000):
        args[9] = eps
        got = words(fn, tuple(args))
        assert got[9] == struct.unpack("<I", bytes(C.c_float(eps)))[0] and got[1] == 63
        direct = fn(*args[:1], 63, *args[2:], None)
        with pytest.raises(B.DfqError) as e:
            B.CallList([(fn, tuple(args))]).run(None)
        assert e.value.status == direct


def test_one_argument_too_many_is_refused():
    for fn, n in ((B.lib().dfq_rms_norm_mx, 20), (B.lib().dfq_quantize_mx, 11)):
        for more in (1, 2, 5):
            with pytest.raises(B.DfqError) as e:
                B.CallList([(fn, (0,) * (n + more))]).run(None)
            assert e.value.status == B.EINVAL
