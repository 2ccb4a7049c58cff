"""The oracle of the microscaled tensors against closed forms, the paper's own codes and another implementation of the element types."""
from fractions import Fraction

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import mx, npfmt


def test_elements_are_the_papers_codes():
    assert mx.magnitudes(mx.MX4).tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    assert mx.magnitudes(mx.MX4)[-1] == npfmt.beta_max(4, 1) / 2
    e4m3 = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(mx.magnitudes(mx.MX8), e4m3) and e4m3[-1] == 448


def test_nearest_code_is_the_types_own_rounding():
    rng = np.random.default_rng(1)
    t = mx.magnitudes(mx.MX8)
    v = np.concatenate((rng.standard_normal(5000) * np.exp(rng.uniform(-8, 6, 5000)), t, -t, (t[1:] + t[:-1]) / 2)).astype(np.float32)
    v = v[np.abs(v) <= 448]
    want = (torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8).numpy()).copy()
    want[want == 0x80] = 0                                       # -0 is not written
    assert np.array_equal(mx.nearest_code(v, mx.MX8), want)
    # the 4-bit ones by hand: every tie, to the even code
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    assert mx.nearest_code(ties, mx.MX4).tolist() == [0, 2, 2, 4, 4, 6, 6]
    assert mx.nearest_code(-ties, mx.MX4).tolist() == [0, 10, 10, 12, 12, 14, 14]
    assert mx.nearest_code([7.99, -100, 0.26, -0.1], mx.MX4).tolist() == [7, 15, 1, 0]


@pytest.mark.parametrize("elem, top", [(mx.MX4, 6), (mx.MX8, 448)])
def test_scale_rules(elem, top):
    s = lambda a, rule: mx.scale_byte(a, elem, rule)
    step = np.nextafter(np.float32(top), np.float32(1e9))
    assert s(top, mx.COVER) == 127 and s(float(step), mx.COVER) == 128 and s(top / 2, mx.COVER) == 126
    power = 4 if elem == mx.MX4 else 256
    assert s(power, mx.FLOOR) == 127 and s(np.nextafter(np.float32(2 * power), np.float32(0)), mx.FLOOR) == 127 and s(2 * power, mx.FLOOR) == 128
    for rule in (mx.COVER, mx.FLOOR):
        assert s(0.0, rule) == 0 and s(2.0 ** -149, rule) == 0 and s(np.inf, rule) == 255 and s(np.nan, rule) == 255
        assert s(float(np.finfo(np.float32).max), rule) <= 253
    # the covering exponent is -f of the rule that the (n, p) codes have, with the element's largest value for beta_max
    for a in (0.013, 1.0, 5.9, 6.1, 447.0, 449.0, 3e4):
        f = max(g for g in range(-40, 41) if Fraction(a) * Fraction(2) ** g <= top)
        assert s(a, mx.COVER) == 127 - f


def test_a_block_by_hand():
    x = np.zeros((1, 34))
    x[0, :4] = [3.0, -1.0, 0.3, 12.0]
    x[0, 32:] = [-0.25, 1e-9]
    codes, scales = mx.quantize(x, mx.MX4, mx.COVER)
    assert scales.tolist() == [[128, 123, 0, 0]]                  # 12 = 6 * 2^1; 0.25 = 4 * 2^-4
    assert codes.shape == (1, 32)
    assert codes[0, :2].tolist() == [3 | 9 << 4, 0 | 7 << 4]       # 1.5, -0.5, 0.15 -> 0, 6
    assert codes[0, 16] == 14 and not codes[0, 17:].any()
    assert mx.values(codes, scales, mx.MX4, 34)[0, [0, 1, 2, 3, 32, 33]].tolist() == [3, -1, 0, 12, -0.25, 0]
    codes, scales = mx.quantize(x, mx.MX4, mx.FLOOR)
    assert scales[0, 0] == 128 and scales[0, 1] == 123
    x[0, 3] = 15.0                                                # floor(log2 15) - 2 = 1: saturates at 12
    codes, scales = mx.quantize(x, mx.MX4, mx.FLOOR)
    assert scales[0, 0] == 128 and mx.values(codes, scales, mx.MX4, 34)[0, 3] == 12
    x[0, 5] = np.nan
    codes, scales = mx.quantize(x, mx.MX8, mx.FLOOR)
    assert scales[0, 0] == 255 and not codes[0, :32].any() and np.isnan(mx.values(codes, scales, mx.MX8, 34)[0, :32]).all()


def test_norm_by_hand():
    s, v = mx.rms_norm([[3.0, 4.0]], [[0.0, 0.0]], [2.0, 1.0], 0.0)
    assert s.tolist() == [[3, 4]] and np.allclose(v, [[6 / np.sqrt(12.5), 4 / np.sqrt(12.5)]], rtol=1e-15)
