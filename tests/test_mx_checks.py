"""What the microscaled calls refuse before anything is launched; no GPU needed (addresses are never read)."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

from paper_1805_07941_amd import binding as B

A = [(i + 1) << 32 for i in range(12)]        # addresses far apart


def quantize(**kw):
    a = dict(x=A[0], ldx=64, dtype=1, rows=3, K=64, codes=A[1], ldc=64, scales=A[2], lds=4, elem=B.MX8, rule=0)
    a.update(kw)
    return B.lib().dfq_quantize_mx(*a.values(), None)


def dequantize(**kw):
    a = dict(codes=A[1], ldc=64, scales=A[2], lds=4, elem=B.MX8, rows=3, K=64, x=A[0], ldx=64, dtype=1)
    a.update(kw)
    return B.lib().dfq_dequantize_mx(*a.values(), None)


OPERANDS = dict(x=A[0], ldx=64, xs=A[1], ldxs=4, ex=B.MX8, w=A[2], ldw=32, ws=A[3], ldws=4, ew=B.MX4, bias=None)


def linear(**kw):
    a = dict(OPERANDS, y=A[4], ldy=16, dtype=1, M=3, N=16, K=64, relu=0)
    a.update(kw)
    return B.lib().dfq_linear_mx(*a.values(), None)


def linear_q(**kw):
    a = dict(OPERANDS, codes=A[4], ldc=32, scales=A[5], lds=4, elem=B.MX8, rule=0, M=3, N=16, K=64, relu=0)
    a.update(kw)
    return B.lib().dfq_linear_mx_q(*a.values(), None)


def norm(**kw):
    a = dict(x=A[0], ldx=64, add=A[1], ldadd=64, sum=A[2], ldsum=64, dtype=1, weight=A[3], wtype=1, eps=1e-6, y=A[4], ldy=64, codes=A[5], ldc=64,
             scales=A[6], lds=4, elem=B.MX8, rule=0, rows=3, K=64)
    a.update(kw)
    return B.lib().dfq_rms_norm_mx(*a.values(), None)


BIG = 1 << 22


@pytest.mark.parametrize("kw, status", [
    (dict(x=None), B.EINVAL), (dict(x=A[0] + 1), B.EINVAL), (dict(dtype=3), B.EINVAL), (dict(dtype=0, x=A[0] + 2), B.EINVAL), (dict(K=0), B.ESHAPE),
    (dict(K=BIG + 1, ldx=2 * BIG, ldc=2 * BIG, lds=BIG), B.EUNSUPPORTED), (dict(rows=1 << 31), B.EUNSUPPORTED), (dict(ldx=63), B.ESHAPE),
    (dict(codes=None), B.EINVAL), (dict(codes=A[1] + 8), B.EINVAL), (dict(ldc=72), B.ESHAPE), (dict(ldc=48), B.ESHAPE), (dict(scales=None), B.EINVAL),
    (dict(scales=A[2] + 2), B.EINVAL), (dict(lds=6), B.ESHAPE), (dict(lds=0), B.ESHAPE), (dict(elem=2), B.EINVAL), (dict(rule=2), B.EINVAL),
    (dict(codes=A[0] + 320), B.EINVAL), (dict(scales=A[1] + 128), B.EINVAL), (dict(scales=A[0] + 380), B.EINVAL),
    (dict(K=33, elem=B.MX4, ldc=16), B.ESHAPE), (dict(K=129, ldx=200, ldc=160), B.ESHAPE), (dict(ldx=1 << 41), B.EUNSUPPORTED)])
def test_quantize_refuses(kw, status):
    assert quantize(**kw) == status


@pytest.mark.parametrize("kw, status", [
    (dict(x=None), B.EINVAL), (dict(x=A[0] + 1), B.EINVAL), (dict(dtype=-1), B.EINVAL), (dict(K=0), B.ESHAPE), (dict(ldx=63), B.ESHAPE), (dict(elem=7), B.EINVAL),
    (dict(codes=A[1] + 4), B.EINVAL), (dict(ldc=56), B.ESHAPE), (dict(scales=None), B.EINVAL), (dict(lds=5), B.ESHAPE), (dict(x=A[1]), B.EINVAL), (dict(x=A[2]), B.EINVAL)])
def test_dequantize_refuses(kw, status):
    assert dequantize(**kw) == status


SHARED = [(dict(x=None), B.EINVAL), (dict(xs=None), B.EINVAL), (dict(w=None), B.EINVAL), (dict(ws=None), B.EINVAL), (dict(x=A[0] + 8), B.EINVAL),
          (dict(ws=A[3] + 1), B.EINVAL), (dict(ex=2), B.EINVAL), (dict(ew=-1), B.EINVAL), (dict(K=0), B.ESHAPE), (dict(N=0), B.ESHAPE), (dict(ldx=48), B.ESHAPE),
          (dict(ldw=24), B.ESHAPE), (dict(ldw=16), B.ESHAPE), (dict(ldxs=2), B.ESHAPE), (dict(ldws=0), B.ESHAPE), (dict(K=65), B.ESHAPE),
          (dict(M=1 << 31), B.EUNSUPPORTED), (dict(bias=A[7] + 2), B.EINVAL), (dict(M=0, K=0), B.ESHAPE)]


@pytest.mark.parametrize("kw, status", SHARED + [
    (dict(y=None), B.EINVAL), (dict(y=A[4] + 1), B.EINVAL), (dict(dtype=4), B.EINVAL), (dict(ldy=15), B.ESHAPE), (dict(y=A[0] + 2), B.EINVAL), (dict(y=A[3]), B.EINVAL),
    (dict(bias=A[7], y=A[7] + 60), B.EINVAL), (dict(N=BIG + 1, ldy=2 * BIG), B.EUNSUPPORTED), (dict(N=0x7fffffff, ldy=1 << 31), B.EUNSUPPORTED)])
def test_linear_refuses(kw, status):
    assert linear(**kw) == status


@pytest.mark.parametrize("kw, status", SHARED + [
    (dict(codes=None), B.EINVAL), (dict(scales=None), B.EINVAL), (dict(codes=A[4] + 8), B.EINVAL), (dict(ldc=16), B.ESHAPE), (dict(lds=3), B.ESHAPE),
    (dict(elem=2), B.EINVAL), (dict(rule=-1), B.EINVAL), (dict(codes=A[2]), B.EINVAL), (dict(scales=A[4] + 64), B.EINVAL), (dict(scales=A[1]), B.EINVAL)])
def test_linear_q_refuses(kw, status):
    assert linear_q(**kw) == status


def variant(which, **kw):
    a = dict(OPERANDS, y=A[4], ldy=16, dtype=1, codes=None, ldc=0, scales=None, lds=0, elem=B.MX8, rule=0, M=3, N=16, K=64, relu=0)
    a.update(kw)
    return B.lib().dfq_linear_mx_variant(which, *a.values(), None)


@pytest.mark.parametrize("which, kw, status", [
    (-1, {}, B.EINVAL), (11, {}, B.EINVAL), (3, dict(codes=A[5], ldc=32, scales=A[6], lds=4), B.EINVAL), (3, dict(y=None), B.EINVAL), (10, dict(ldy=15), B.ESHAPE),
    (2, dict(y=None, codes=A[5], ldc=32, scales=A[6], lds=4), B.EUNSUPPORTED), (10, dict(ldx=(1 << 22) + 16), B.EUNSUPPORTED),
    (3, dict(ldws=(1 << 22) + 4), B.EUNSUPPORTED), (0, dict(y=None, codes=A[5], ldc=16, scales=A[6], lds=4), B.ESHAPE)])
def test_linear_variant_refuses(which, kw, status):
    assert variant(which, **kw) == status


@pytest.mark.parametrize("kw, status", [
    (dict(x=None), B.EINVAL), (dict(y=None, codes=None), B.EINVAL), (dict(scales=None), B.EINVAL), (dict(dtype=3), B.EINVAL), (dict(wtype=2), B.EINVAL),
    (dict(eps=-1.0), B.EINVAL), (dict(eps=float("nan")), B.EINVAL), (dict(eps=float("inf")), B.EINVAL), (dict(K=0), B.ESHAPE), (dict(ldadd=60), B.ESHAPE),
    (dict(ldsum=1), B.ESHAPE), (dict(ldy=63), B.ESHAPE), (dict(ldx=0), B.ESHAPE), (dict(weight=A[3] + 1), B.EINVAL), (dict(wtype=0, weight=A[3] + 2), B.EINVAL),
    (dict(add=A[1] + 1), B.EINVAL), (dict(sum=A[0] + 2), B.EINVAL), (dict(sum=A[0], ldsum=128), B.EINVAL), (dict(sum=A[1], ldsum=72), B.EINVAL),
    (dict(sum=A[4]), B.EINVAL), (dict(y=A[0]), B.EINVAL), (dict(codes=A[1]), B.EINVAL), (dict(scales=A[4]), B.EINVAL), (dict(sum=A[3]), B.EINVAL),
    (dict(sum=A[0], add=A[0] + 64), B.EINVAL), (dict(elem=3), B.EINVAL), (dict(rule=5), B.EINVAL), (dict(rows=1 << 31), B.EUNSUPPORTED)])
def test_norm_refuses(kw, status):
    assert norm(**kw) == status


@pytest.mark.parametrize("call, kw", [
    (quantize, dict(ldx=1 << 40)), (quantize, dict(ldc=1 << 40)), (quantize, dict(lds=1 << 40)), (dequantize, dict(ldx=1 << 40)), (linear, dict(ldx=1 << 40)),
    (linear, dict(ldy=1 << 40)), (linear_q, dict(ldc=1 << 40)), (norm, dict(ldadd=1 << 40)), (norm, dict(ldsum=1 << 40)), (norm, dict(ldy=1 << 40))])
def test_rows_whose_addresses_leave_64_bits(call, kw):
    """2^24 + 1 of them 2^40 apart: a distance that wraps around is no check of what lies where."""
    rows = "M" if call in (linear, linear_q) else "rows"
    assert call(**kw, **{rows: (1 << 24) + 1}) == B.EUNSUPPORTED


def test_nothing_to_do():
    assert quantize(rows=0, x=None, codes=None, scales=None) == B.OK and dequantize(rows=0, x=None) == B.OK
    assert linear(M=0, x=None, y=None) == B.OK and linear_q(M=0, codes=None) == B.OK and norm(rows=0, x=None, y=None, codes=None) == B.OK


def test_records_of_the_calls():
    """Each as one call of a list: refused by its own function, a float argument by its bits."""
    L = B.lib()
    lists = [(L.dfq_quantize_mx, (A[0], 63, 1, 3, 64, A[1], 64, A[2], 4, 1, 0), B.ESHAPE),
             (L.dfq_dequantize_mx, (A[1], 64, A[2], 4, 1, 3, 64, A[0], 63, 1), B.ESHAPE),
             (L.dfq_linear_mx, tuple(OPERANDS.values()) + (A[4], 15, 1, 3, 16, 64, 0), B.ESHAPE),
             (L.dfq_linear_mx_q, tuple(OPERANDS.values()) + (A[4], 16, A[5], 4, 1, 0, 3, 16, 64, 0), B.ESHAPE)]
    for eps, status in ((float("nan"), B.EINVAL), (-0.5, B.EINVAL), (1e-6, B.ESHAPE)):
        lists.append((L.dfq_rms_norm_mx, (A[0], 63, None, 0, None, 0, 1, None, 1, eps, A[4], 64, None, 0, None, 0, 1, 0, 3, 64), status))
    for fn, args, status in lists:
        assert fn(*args, None) == status
        with pytest.raises(B.DfqError, match=fn.__name__) as e:
            B.CallList([(fn, args)]).run(None)
        assert e.value.status == status


def test_a_record_of_a_whole_number_where_a_float_belongs():
    """0x7f800000 as a float's bits would be an infinity and refused; as a number it is an eps like any other."""
    fn = B.lib().dfq_rms_norm_mx
    args = (A[0], 63, None, 0, None, 0, 1, None, 1, 0x7f800000, A[4], 64, None, 0, None, 0, 1, 0, 3, 64)
    assert fn(*args, None) == B.ESHAPE
    with pytest.raises(B.DfqError) as e:
        B.CallList([(fn, args)]).run(None)
    assert e.value.status == B.ESHAPE


def test_tensors_on_the_host_are_refused():
    x = torch.zeros(2, 64)
    q = B.MxTensor.empty(2, 64, B.MX8, "cpu")
    for call in (lambda: B.quantize_mx(x), lambda: B.dequantize_mx(q), lambda: B.linear_mx(q, q), lambda: B.linear_mx_q(q, q), lambda: B.rms_norm_mx(x)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
