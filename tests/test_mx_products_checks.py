"""What the products' choice of accuracy accepts and refuses before anything is launched; no GPU needed (addresses are never read)."""
import pytest

torch = pytest.importorskip("torch")

from paper_1805_07941_amd import binding as B
from test_mx_checks import A, variant


@pytest.mark.parametrize("which, kw, status", [
    (15, {}, B.EINVAL), (27, {}, B.EINVAL), (32, {}, B.EINVAL), (48, {}, B.EINVAL), (-16, {}, B.EINVAL), (16, dict(y=None), B.EINVAL), (26, dict(ldy=15), B.ESHAPE),
    (18, dict(y=None, codes=A[5], ldc=32, scales=A[6], lds=4), B.EUNSUPPORTED), (26, dict(ldx=(1 << 22) + 16), B.EUNSUPPORTED)])
def test_aligned_products_refuse(which, kw, status):
    assert B.LINEAR_ALIGNED == 16 and variant(which, **kw) == status


def test_nothing_to_do():
    for which in range(11):
        assert variant(which + B.LINEAR_ALIGNED, M=0, x=None, y=None) == B.OK
