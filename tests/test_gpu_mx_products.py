"""Products on microscaled operands where they are hardest to hold: sums that cancel, blocks that hold no numbers, scales at the ends of their
range, long reductions through the tile kernels.  Bounds as in test_gpu_mx.py: float32's step u = 2^-24 and half a step of the result's type."""
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


def converted_within(B, q, want, err, elem, rule):
    """A converted result [M, N] against the sums it stands for, each known to within err."""
    M, N = want.shape
    nb = -(-N // 32)
    codes, scales = host(q.codes), host(q.scales)
    wide, ewide = (np.pad(v, ((0, 0), (0, nb * 32 - N))) for v in (want, err))
    amax, slack = np.abs(wide).reshape(M, nb, 32).max(2), ewide.reshape(M, nb, 32).max(2)
    for m in range(M):
        for k in range(nb):
            lo, hi = (mx.scale_byte(max(a, 0.0), ELEM[elem], rule) for a in (amax[m, k] - slack[m, k], amax[m, k] + slack[m, k]))
            assert lo <= scales[m, k] <= hi, (m, k, scales[m, k], lo, hi)
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


@pytest.mark.parametrize("variant", VARIANTS)
@pytest.mark.parametrize("ex, ew", PAIRS)
def test_aligned_products(B, ex, ew, variant):
    """What a caller asks for by LINEAR_ALIGNED: within what the alignment of eight products adds; on 4-bit operands nothing changes."""
    for M, N, K in ALIGNED_SHAPES:
        (x, w, b), (vx, vw, vb) = products(B, rng_of("aligned", ex, ew, M, N, K), M, N, K, ex, ew, True)
        want, err = mx.linear(vx, vw, vb), product_bound(vx, vw, vb, (ex, ew), False)
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
