"""The root-mean-square norm where float32 is short of range or of digits: rows of values far apart, rows of millions of values."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import mx
from test_gpu_mx import B, DEV, HALF, NORM_U, TYPES, host, rng_of  # noqa: F401 (B is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K", [20, 500, 2000, 4096, 9000, 40000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_small_values_beside_large_ones(B, dtype, K):
    """A row's first value sets its mean square, the others are far smaller: what they become is as near as in any other row."""
    rng = rng_of("apart", dtype, K)
    pairs = [(51, -75), (52, -72), (60, -60), (100, -20), (126, 3), (127, -20), (50, -73), (64, -61), (-45, -149), (-60, -120), (-41, -140), (0, -100)]
    x = torch.from_numpy(np.clip(np.abs(rng.standard_normal((len(pairs), K))) + 0.1, 0, 1.9) * np.exp2(np.array([p[1] for p in pairs], np.float64))[:, None]).to(TYPES[dtype])
    x[:, 0] = torch.from_numpy(np.exp2(np.array([p[0] for p in pairs], np.float64))).to(TYPES[dtype])
    x[0, 2:] = 0
    for eps in (0.0, 1e-30):
        _, v = mx.rms_norm(x.float().numpy(), None, None, eps)
        q, y, _ = B.rms_norm_mx(x.to(DEV), None, eps, want_y=True)
        err = NORM_U * np.abs(v)
        # the value is rounded as a float32 first, and below 2^-126 to a multiple of 2^-149 before it is rounded to its type
        tol = err + HALF[dtype] * (np.abs(v) + err) + 2.0 ** (-149 if dtype == "f32" else -133)
        ok = np.abs(host(y) - v) <= tol
        assert ok.all(), (eps, np.argwhere(~ok)[:4], [(host(y)[tuple(i)], v[tuple(i)]) for i in np.argwhere(~ok)[:4]])
        if dtype == "f32":
            same = B.quantize_mx(y)
            assert torch.equal(q.codes, same.codes) and torch.equal(q.scales, same.scales)


@pytest.mark.parametrize("value", [1.05, 1.1, 1.3, 3.3])
@pytest.mark.parametrize("K", [40000, 1 << 20, (1 << 22) - 5])
def test_long_rows_of_one_value(B, K, value):
    """Every addition of equal squares rounds the same way: a sum of thousands by one thread must not gather that."""
    x = torch.full((2, K), value, device=DEV)
    x[1] = -value
    for eps in (0.0, 1e-3):
        _, y, _ = B.rms_norm_mx(x, None, eps, elem=None, want_y=True)
        d = float(np.float32(value))
        v = d / np.sqrt(d * d + float(np.float32(eps)))
        off = np.abs(np.abs(host(y)) - v).max() / v
        assert off <= NORM_U, off / NORM_U * 64


@pytest.mark.parametrize("K", [1 << 15, 3 << 20, (1 << 22) - 5])
def test_a_smallest_value_among_zeros(B, K):
    """One value of 1 to 5 times 2^-149 in a long row: the mean square is far below float32's smallest numbers, its root is not."""
    x = torch.zeros(3, K, device=DEV)
    for r, n in enumerate((1, 3, 5)):
        x[r, 7 * r] = float(n * 2.0 ** -149)
    _, y, _ = B.rms_norm_mx(x, None, 0.0, elem=None, want_y=True)
    y = host(y)
    for r in range(3):
        assert abs(y[r, 7 * r] / np.sqrt(K) - 1) <= NORM_U, (r, abs(y[r, 7 * r] / np.sqrt(K) - 1) / NORM_U * 64)
    assert np.count_nonzero(y) == 3
