"""The tile kernels of the products on what only long reductions and whole tiles reach: rings of scales that wrap, results that go past the
cache, converted results of both element types by both rules, the choice between them."""
import functools
import re

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import mx
from test_gpu_mx import B, DEV, ELEM, HALF, PAIRS, TYPES, U, host, on_gpu, operand, product_bound, products, rng_of  # noqa: F401 (B is a fixture)
from test_gpu_mx_products import converted_within

pytestmark = pytest.mark.gpu

TILES = range(6, 11)


def results_within(B, x, w, b, want, errs, variant, elems=(4, 8)):
    """Every type of result of one kernel, and both ways to take 8-bit operands.  Converted results are those of the float32 ones."""
    exact, aligned = errs
    for how, err in ((0, exact), (B.LINEAR_ALIGNED, aligned)):
        if how and x.elem == w.elem == B.MX4:
            continue
        for out in TYPES:
            y = host(B.linear_mx(x, w, b, dtype=TYPES[out], variant=variant + how))
            tol = err + HALF[out] * (np.abs(want) + err) + (2.0 ** -25 if out == "f16" else 0)
            ok = (np.abs(y - want) <= tol) | ((out == "f16") & np.isinf(y) & (np.abs(want) + tol > 65504))
            assert ok.all(), (variant, how, out, np.argwhere(~ok)[:4])
        f32 = B.linear_mx(x, w, b, dtype=torch.float32, variant=variant + how)
        for elem in elems:
            for rule in (mx.COVER, mx.FLOOR):
                q = B.linear_mx_q(x, w, b, ELEM[elem], rule, variant=variant + how)
                converted_within(B, q, want, err, elem, rule)
                same = B.quantize_mx(f32, ELEM[elem], rule)
                assert torch.equal(q.codes, same.codes) and torch.equal(q.scales, same.scales), (variant, how, elem, rule)


@functools.lru_cache(maxsize=None)
def case(B, ex, ew, M, N, K, spread):
    """Operands whose scales are 2^spread apart, a bias; the sums with and without it, and what they may be off by."""
    rng = rng_of("tiles", ex, ew, M, N, K)
    qx, qw = (operand(rng, rows, K, e, spread) for rows, e in ((M, ex), (N, ew)))
    b = rng.standard_normal(N).astype(np.float32)
    vx, vw = mx.values(*qx, ELEM[ex], K), mx.values(*qw, ELEM[ew], K)
    errs = [product_bound(vx, vw, b, (ex, ew), e) for e in (True, False)]
    return (on_gpu(B, qx, ex, K), on_gpu(B, qw, ew, K), torch.from_numpy(b).to(DEV)), (mx.linear(vx, vw, b), mx.linear(vx, vw)), errs


@pytest.mark.parametrize("variant", [1, 3, 4, 5, *TILES])
@pytest.mark.parametrize("ex, ew", PAIRS)
def test_rings_of_scales_that_wrap(B, ex, ew, variant):
    """K of nine chunks of scales, the last one short: each slot of a ring of four or eight is read with another chunk's scales."""
    operands, (want, _), errs = case(B, ex, ew, 70, 140, 4470, 12)
    results_within(B, *operands, want, errs, variant)


@pytest.mark.parametrize("variant", TILES)
@pytest.mark.parametrize("ex, ew", PAIRS)
def test_whole_tiles(B, ex, ew, variant):
    """Results whose rows are whole cache lines: tiles without an edge, of 256 x 256 past the cache, with and without a bias."""
    (x, w, b), (want, plain), errs = case(B, ex, ew, 512, 512, 320, 6)
    results_within(B, x, w, b, want, errs, variant)
    results_within(B, x, w, None, plain, errs, variant, elems=(8,))


@pytest.mark.parametrize("ex, ew, M, N, K, tile", [(4, 4, 700, 900, 1000, (64, 64)), (8, 4, 1100, 1100, 300, (64, 128)), (8, 8, 2048, 2304, 256, (128, 128)),
                                                   (4, 4, 2048, 2048, 512, (128, 128)), (4, 4, 4096, 4096, 256, (256, 256))])
def test_calls_that_choose_tiles(B, ex, ew, M, N, K, tile):
    """The choice by the call itself: these sizes run tiles, and their results are those sums."""
    (x, w, _), (vx, vw, _) = products(B, rng_of("choice", ex, ew, M), M, N, K, ex, ew, False)
    want, total = torch.from_numpy(vx).to(DEV) @ torch.from_numpy(vw).to(DEV).t(), torch.from_numpy(np.abs(vx)).to(DEV) @ torch.from_numpy(np.abs(vw)).to(DEV).t()
    err = (K + 8) * U * total
    for out in TYPES:
        y = B.linear_mx(x, w, dtype=TYPES[out]).double()
        tol = err + HALF[out] * (want.abs() + err) + (2.0 ** -25 if out == "f16" else 0)
        assert (((y - want).abs() <= tol) | (y.isinf() & (want.abs() + tol > 65504) & (out == "f16"))).all()
    f32 = B.linear_mx(x, w, dtype=torch.float32)
    for elem in (B.MX4, B.MX8):
        q, same = B.linear_mx_q(x, w, elem=elem), B.quantize_mx(f32, elem)
        assert torch.equal(q.codes, same.codes) and torch.equal(q.scales, same.scales)
    torch.cuda.synchronize()
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA]) as prof:
        B.linear_mx(x, w)
        torch.cuda.synchronize()
    names = [e.name for e in prof.events() if e.device_type == torch.autograd.DeviceType.CUDA and "linear_mx" in e.name]
    if not names:
        pytest.skip("the device's activity is not recorded here")
    assert len(names) == 1 and "tiles" in names[0] and re.search(rf"\b{tile[0]}, {tile[1]},|Li{tile[0]}ELi{tile[1]}E", names[0]), names
