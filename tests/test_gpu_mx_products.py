"""Products on microscaled operands where they are hardest to hold: sums that cancel, blocks that hold no numbers, scales at the ends of their
range, long reductions through the tile kernels.  Bounds as in test_gpu_mx.py: float32's step u = 2^-24 and half a step of the result's type."""
import functools

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import mx
from test_gpu_mx import B, DEV, ELEM, HALF, PAIRS, TYPES, U, host, on_gpu, product_bound, products, rng_of, steps_of  # noqa: F401 (B is a fixture)

pytestmark = pytest.mark.gpu

VARIANTS = range(0, 11)
HALF_A_BLOCK = 2                    # the kernel whose workgroups have half of a block: no converted results


def codes_of(v, elem):
    """Values that are elements, at scale 1 -> what the tensors hold."""
    rows, K = v.shape
    full = np.zeros((rows, -(-K // 32) * 32))
    full[:, :K] = v
    c = mx.nearest_code(full, ELEM[elem])
    scales = np.zeros((rows, -(-(-(-K // 32)) // 4) * 4), np.uint8)
    scales[:, :-(-K // 32)] = 127
    return (c[:, 0::2] | c[:, 1::2] << 4 if elem == 4 else c), scales


def scale_bytes(amax, elem, rule):
    """oracle/mx.py's scale_byte for an array of finite magnitudes."""
    powers, top = np.exp2(np.arange(255.0) - 127), mx.magnitudes(ELEM[elem])[-1]
    if rule == mx.COVER:
        return np.searchsorted(top * powers, amax)
    return np.maximum(np.searchsorted(2.0 ** np.floor(np.log2(top)) * powers, amax, side="right") - 1, 0)


def test_scale_bytes_are_the_oracles():
    rng = rng_of("bytes")
    v = np.concatenate(([0.0, 6.0, 448.0, 4.0, 256.0, 8.0, 512.0, 2.0 ** -149], np.exp2(rng.uniform(-140, 120, 40))))
    for elem in (4, 8):
        for rule in (mx.COVER, mx.FLOOR):
            assert scale_bytes(v, elem, rule).tolist() == [mx.scale_byte(a, ELEM[elem], rule) for a in v]


def converted_within(B, q, want, err, elem, rule):
    """A converted result [M, N] against the sums it stands for, each known to within err."""
    M, N = want.shape
    nb = -(-N // 32)
    codes, scales = host(q.codes), host(q.scales)
    wide, ewide = (np.pad(v, ((0, 0), (0, nb * 32 - N))) for v in (want, err))
    amax, slack = np.abs(wide).reshape(M, nb, 32).max(2), ewide.reshape(M, nb, 32).max(2)
    lo, hi = (scale_bytes(np.maximum(a, 0), elem, rule) for a in (amax - slack, amax + slack))
    assert ((lo <= scales[:, :nb]) & (scales[:, :nb] <= hi)).all()
    assert not scales[:, nb:].any()
    got = mx.values(codes, scales, ELEM[elem], nb * 32)
    assert not got[:, N:].any()
    scale = np.exp2(scales[:, :nb].astype(np.float64) - 127).repeat(32, 1)
    top = mx.magnitudes(ELEM[elem])[-1] * scale
    near = np.clip(wide, -top, top)
    half = np.maximum(steps_of(np.abs(near) + ewide, scale, elem), steps_of(near, scale, elem))
    ok = np.abs(got - near) <= ewide + half
    assert ok.all(), np.argwhere(~ok)[:4]


def cancelling(rng, M, N, K, ex, ew):
    """Of eight consecutive k the first two products are the largest there are and cancel; the others are 2^-10 to 2^-20 of them."""
    def side(rows, elem, signs):
        t = mx.magnitudes(ELEM[elem])
        big, small = t[-4:], t[1:3] if elem == 4 else t[56:80] if ex == ew else t[1:16]
        v = rng.choice(small, (rows, K)) * rng.choice([-1, 1], (rows, K))
        for s in range(0, K - 1, 8):
            v[:, s] = rng.choice(big, rows)
            v[:, s + 1] = v[:, s] * signs
        return v
    return side(M, ex, 1), side(N, ew, -1)


@pytest.mark.parametrize("M, N, K", [(1, 40, 32), (5, 33, 40), (40, 70, 64), (130, 140, 96), (300, 257, 32)])
@pytest.mark.parametrize("ex, ew", PAIRS)
def test_sums_that_cancel(B, ex, ew, M, N, K):
    """Products and sums are float32's whatever the result's type: a sum is off by steps of the products it adds, (K + 8) u of their
    magnitudes' sum, and by half a step of its own type."""
    rng = rng_of("cancel", ex, ew, M, N, K)
    vx, vw = cancelling(rng, M, N, K, ex, ew)
    x, w = on_gpu(B, codes_of(vx, ex), ex, K), on_gpu(B, codes_of(vw, ew), ew, K)
    want = mx.linear(vx, vw)
    err = product_bound(vx, vw, None, (ex, ew), True)
    for variant in VARIANTS:
        for out in TYPES:
            y = host(B.linear_mx(x, w, dtype=TYPES[out], variant=variant))
            tol = err + HALF[out] * (np.abs(want) + err) + (2.0 ** -25 if out == "f16" else 0)
            ok = np.abs(y - want) <= tol
            assert ok.all(), (variant, out, np.argwhere(~ok)[:4], (np.abs(y - want) / tol).max())
        if variant != HALF_A_BLOCK:
            for elem, rule in ((8, mx.COVER), (4, mx.FLOOR)):
                converted_within(B, B.linear_mx_q(x, w, elem=ELEM[elem], rule=rule, variant=variant), want, err, elem, rule)


ALIGNED_SHAPES = [(1, 1, 1), (3, 35, 97), (16, 32, 300), (33, 65, 513), (70, 100, 1025), (130, 140, 1600), (257, 300, 700)]


@functools.lru_cache(maxsize=None)
def aligned_case(B, ex, ew, M, N, K):
    gpu, (vx, vw, vb) = products(B, rng_of("aligned", ex, ew, M, N, K), M, N, K, ex, ew, True)
    return gpu, mx.linear(vx, vw, vb), product_bound(vx, vw, vb, (ex, ew), False)


@pytest.mark.parametrize("variant", VARIANTS)
@pytest.mark.parametrize("ex, ew", PAIRS)
def test_aligned_products(B, ex, ew, variant):
    """What a caller asks for by LINEAR_ALIGNED: within what the alignment of eight products adds; on 4-bit operands nothing changes."""
    for M, N, K in ALIGNED_SHAPES:
        (x, w, b), want, err = aligned_case(B, ex, ew, M, N, K)
        for out in TYPES:
            got = B.linear_mx(x, w, b, dtype=TYPES[out], variant=variant + B.LINEAR_ALIGNED)
            tol = err + HALF[out] * (np.abs(want) + err) + (2.0 ** -25 if out == "f16" else 0)
            ok = (np.abs(host(got) - want) <= tol) | ((out == "f16") & np.isinf(host(got)) & (np.abs(want) + tol > 65504))
            assert ok.all(), (M, N, K, out, np.argwhere(~ok)[:4])
            if ex == ew == 4:
                assert torch.equal(got, B.linear_mx(x, w, b, dtype=TYPES[out], variant=variant))
        if variant != HALF_A_BLOCK:
            for elem, rule in ((8, mx.COVER), (4, mx.FLOOR)):
                q = B.linear_mx_q(x, w, b, ELEM[elem], rule, variant=variant + B.LINEAR_ALIGNED)
                converted_within(B, q, want, err, elem, rule)


def test_aligned_products_in_a_list_of_calls(B):
    """One call of a list like any other."""
    (x, w, b), _ = products(B, rng_of("list"), 9, 40, 300, 8, 4, True)
    want = B.linear_mx(x, w, b, variant=B.LINEAR_ALIGNED)
    y = torch.full_like(want, 7.0)
    at = lambda q: (q.codes.data_ptr(), q.codes.stride(0), q.scales.data_ptr(), q.scales.stride(0), q.elem)
    args = (B.LINEAR_ALIGNED, *at(x), *at(w), b.data_ptr(), y.data_ptr(), 40, 1, None, 0, None, 0, 0, 0, 9, 40, 300, 0)
    B.CallList([(B.lib().dfq_linear_mx_variant, args)]).run(torch.cuda.current_stream().cuda_stream)
    assert torch.equal(y, want)


def at_scales(rng, rows, K, elem, scale):
    """Codes of every kind but NaN in blocks of one scale."""
    codes = rng.integers(0, 256, (rows, K * elem // 8), dtype=np.uint8)
    if elem == 8:
        codes[(codes & 0x7f) == 0x7f] = 0x38
    return codes, np.full((rows, -(-K // 128) * 4), scale, np.uint8)


@pytest.mark.parametrize("sx, sw", [(0, 240), (1, 235), (3, 240), (8, 230), (240, 0), (240, 3), (246, 6), (230, 8), (4, 246)])
@pytest.mark.parametrize("ex, ew", PAIRS)
def test_scales_at_the_ends_of_their_range(B, ex, ew, sx, sw):
    """One operand's blocks with the smallest scales, the other's with large ones, and the other way round: the sums are ordinary numbers.
    As a bfloat16 an element of 8 bits times its scale is a multiple of 2^-133, half of which is what it may be off by below scale byte 3."""
    M, N, K = 66, 70, 160
    rng = rng_of("ends", ex, ew, sx, sw)
    qx, qw = at_scales(rng, M, K, ex, sx), at_scales(rng, N, K, ew, sw)
    vx, vw = mx.values(*qx, ELEM[ex], K), mx.values(*qw, ELEM[ew], K)
    x, w = on_gpu(B, qx, ex, K), on_gpu(B, qw, ew, K)
    want = mx.linear(vx, vw)
    exact, aligned = (product_bound(vx, vw, None, (ex, ew), e) for e in (True, False))
    if 8 in (ex, ew):
        exact = exact + (2.0 ** -134 * np.abs(vw).sum(1) if ex == 8 and sx < 3 else 0) + (2.0 ** -134 * np.abs(vx).sum(1)[:, None] if ew == 8 and sw < 3 else 0)
    for variant in VARIANTS:
        for how, err in ((0, exact), (B.LINEAR_ALIGNED, aligned)):
            for out in TYPES:
                y = host(B.linear_mx(x, w, dtype=TYPES[out], variant=variant + how))
                tol = err + HALF[out] * (np.abs(want) + err) + (2.0 ** -25 if out == "f16" else 0)
                with np.errstate(invalid="ignore"):
                    ok = (np.abs(y - want) <= tol) | ((out == "f16") & np.isinf(y) & (np.abs(want) + tol > 65504))
                assert ok.all(), (variant, how, out, np.argwhere(~ok)[:4], np.nanmax(np.abs(y - want) / tol))


@pytest.mark.parametrize("ex, ew", [(8, 4), (8, 8), (4, 8)])
def test_elements_beyond_float32(B, ex, ew):
    """2^128 and above, which no conversion of float32 values writes but for values next to it: infinite where elements are taken as
    bfloat16, numbers where they are aligned.  Rows without such elements are what they are."""
    M, N, K = 20, 40, 96
    rng = rng_of("beyond", ex, ew)
    flip = ex == 4                                       # the operand with the large scales is the 8-bit one
    big, other = at_scales(rng, N if flip else M, K, 8, 250), at_scales(rng, M if flip else N, K, ew if not flip else ex, 10)
    eo = ex if flip else ew
    big[0][:] &= 0x87                                    # below 2^-5: subnormal elements
    big[0][::2, 33] = 0x7e                               # 448 * 2^123
    zero = (other[0] & 0x7f) == 0 if eo == 8 else True
    other[0][...] = np.where(zero, other[0] | (1 if eo == 8 else 0x11), other[0])                  # nothing is multiplied by zero
    values = mx.values(*big, mx.MX8, K), mx.values(*other, ELEM[eo], K)
    vx, vw = (values[1], values[0]) if flip else values
    b, o = on_gpu(B, big, 8, K), on_gpu(B, other, eo, K)
    x, w = (o, b) if flip else (b, o)
    want, beyond = mx.linear(vx, vw), np.zeros((M, N), bool)
    beyond[(slice(None), slice(None, None, 2)) if flip else slice(None, None, 2)] = True
    exact, aligned = (product_bound(vx, vw, None, (ex, ew), e) for e in (True, False))
    for variant in VARIANTS:
        y = host(B.linear_mx(x, w, dtype=torch.float32, variant=variant))
        assert not np.isfinite(y[beyond]).any() and (np.abs(y - want) <= exact + U * np.abs(want))[~beyond].all(), variant
        y = host(B.linear_mx(x, w, dtype=torch.float32, variant=variant + B.LINEAR_ALIGNED))
        assert (np.abs(y - want) <= aligned + U * np.abs(want)).all(), variant


@pytest.mark.parametrize("ex, ew", PAIRS)
def test_blocks_that_hold_no_numbers(B, ex, ew):
    """A NaN block as the converter writes it, scale byte 255 over zero codes: every sum that reads it is NaN, the others are what they
    were, by every kernel and in every type; against values, zeros and another such block."""
    M, N, K = 70, 72, 416
    rng = rng_of("nan blocks", ex, ew)
    vx, vw = rng.standard_normal((M, K)).astype(np.float32), rng.standard_normal((N, K)).astype(np.float32)
    vx[3, 40], vx[66, 0], vx[67, K - 1] = np.nan, np.inf, -np.inf
    vw[7, 200], vw[70, K - 1], vw[71, 0] = np.nan, -np.inf, np.inf
    vx[20], vw[30] = 0, 0
    x, w = B.quantize_mx(torch.from_numpy(vx).to(DEV), ELEM[ex]), B.quantize_mx(torch.from_numpy(vw).to(DEV), ELEM[ew])
    assert (host(x.scales)[[3, 66, 67], [1, 0, 12]] == 255).all() and not host(x.codes)[3, ex * 4:ex * 8].any()
    clean_x, clean_w = vx.copy(), vw.copy()
    clean_x[[3, 66, 67]], clean_w[[7, 70, 71]] = 0, 0
    cx, cw = B.quantize_mx(torch.from_numpy(clean_x).to(DEV), ELEM[ex]), B.quantize_mx(torch.from_numpy(clean_w).to(DEV), ELEM[ew])
    bad = np.zeros((M, N), bool)
    bad[[3, 66, 67]], bad[:, [7, 70, 71]] = True, True
    spoilt = np.stack([bad[:, k:k + 32].any(1) for k in range(0, N, 32)], 1).repeat(32, 1)[:, :N]
    for variant in (*VARIANTS, B.LINEAR_ALIGNED, *(v + B.LINEAR_ALIGNED for v in VARIANTS[1:])):
        for out in TYPES:
            for relu in (False, True):
                y, clean = (host(B.linear_mx(a, b, None, relu, TYPES[out], variant=variant)) for a, b in ((x, w), (cx, cw)))
                assert np.array_equal(np.isnan(y), bad), (variant, out, relu)
                assert np.array_equal(y[~bad], clean[~bad]), (variant, out, relu)
        if variant & 15 != HALF_A_BLOCK:
            for elem in (4, 8):
                assert np.array_equal(np.isnan(host(B.dequantize_mx(B.linear_mx_q(x, w, elem=ELEM[elem], relu=True, variant=variant)))), spoilt), (variant, elem)
