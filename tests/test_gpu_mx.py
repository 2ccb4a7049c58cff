"""GPU parity of the microscaled operators with their oracle: conversions byte for byte, products and norms within bounds that follow from
float32's step u = 2^-24, from what the matrix instructions keep (csrc/mx_linear.hpp) and from half a step of the result's type."""
import functools
import zlib

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import mx

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
ELEM = {4: mx.MX4, 8: mx.MX8}


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1805_07941_amd import binding
    binding.lib()
    return binding


def rng_of(*case):
    return np.random.default_rng(zlib.crc32(repr(case).encode()))


def host(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def mixed_values(rng, rows, K):
    """Rows whose blocks have magnitudes from 2^-40 to 2^30, with zeros and blocks of zeros among them."""
    v = rng.standard_normal((rows, K)) * np.exp2(rng.integers(-40, 30, (rows, -(-K // 32))).repeat(32, 1)[:, :K])
    v[rng.random((rows, K)) < 0.05] = 0
    v[:, 32:64] *= rng.random((rows, 1)) < 0.7
    return v


def strided(t, how):
    """The same values in rows of another distance or alignment."""
    if how == "dense":
        return t
    pad, off = {"wide": (16, 0), "odd": (3, 1)}[how]
    room = torch.full((t.shape[0], t.shape[1] + pad), 7.0, dtype=t.dtype, device=t.device)
    room[:, off:off + t.shape[1]] = t
    return room[:, off:off + t.shape[1]]


def same_tensor(q, want, K):
    codes, scales = want
    assert np.array_equal(host(q.scales), scales)
    assert np.array_equal(host(q.codes), codes)


@pytest.mark.parametrize("how", ["dense", "wide", "odd"])
@pytest.mark.parametrize("rows, K", [(1, 1), (3, 31), (2, 32), (5, 33), (7, 100), (4, 128), (1, 1000), (130, 257), (9, 2048)])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_quantize_every_byte(B, dtype, rows, K, how):
    rng = rng_of(dtype, rows, K, how)
    v = mixed_values(rng, rows, K) if dtype != "f16" else rng.standard_normal((rows, K)) * np.exp2(rng.integers(-20, 8, (rows, 1)))
    t = torch.from_numpy(v).to(TYPES[dtype])
    for elem in (4, 8):
        for rule in (mx.COVER, mx.FLOOR):
            q = B.quantize_mx(strided(t.to(DEV), how), ELEM[elem], rule)
            want = mx.quantize(host(t), ELEM[elem], rule)
            same_tensor(q, want, K)
            for out in TYPES:
                back = B.dequantize_mx(q, TYPES[out])
                assert torch.equal(back.cpu(), torch.from_numpy(mx.values(*want, ELEM[elem], K)).to(TYPES[out]))


@pytest.mark.parametrize("elem", [4, 8])
def test_quantize_around_every_boundary(B, elem):
    """Halfway points of neighbouring elements and their neighbours in float32, at scales from the smallest to the largest."""
    t = mx.magnitudes(ELEM[elem])
    edge = np.concatenate((t, (t[1:] + t[:-1]) / 2)).astype(np.float32)
    edge = np.concatenate((edge, np.nextafter(edge, np.float32(0)), np.nextafter(edge, np.float32(1e9))))
    edge = np.concatenate((edge, -edge))
    edge = edge[np.abs(edge) <= t[-1]]
    rows = []
    for e in (-127, -126, -125, -100, -30, 0, 5, 60, 110):
        v = np.pad(edge, (0, -len(edge) % 31)).reshape(-1, 31)
        # one value fixes each block's scale
        v = np.concatenate((np.full((len(v), 1), t[-1]), v), 1).reshape(1, -1)
        rows.append(np.ldexp(v.astype(np.float64), e).astype(np.float32))
    x = np.concatenate(rows)
    for rule in (mx.COVER, mx.FLOOR):
        same_tensor(B.quantize_mx(torch.from_numpy(x).to(DEV), ELEM[elem], rule), mx.quantize(x, ELEM[elem], rule), x.shape[1])


@pytest.mark.parametrize("elem", [4, 8])
def test_quantize_what_is_no_number(B, elem):
    x = np.ones((8, 96), np.float32)
    x[0, 5], x[1, 40], x[2, 95], x[3, 0] = np.nan, np.inf, -np.inf, 3.4e38
    x[4, :32], x[5, :32], x[6, :32] = 2.0 ** -149, -2.0 ** -130, np.float32(2.0 ** -126) * 5
    x[7, :] = -0.0
    for rule in (mx.COVER, mx.FLOOR):
        q = B.quantize_mx(torch.from_numpy(x).to(DEV), ELEM[elem], rule)
        want = mx.quantize(x, ELEM[elem], rule)
        same_tensor(q, want, 96)
        values = torch.from_numpy(mx.values(*want, ELEM[elem], 96)).float()        # (3.4e38 rounds to 2^128: infinity in float32)
        assert np.array_equal(host(B.dequantize_mx(q)), host(values), equal_nan=True)


@pytest.mark.parametrize("elem", [4, 8])
@pytest.mark.parametrize("out", list(TYPES))
def test_dequantize_every_code_at_every_scale(B, elem, out):
    codes = np.tile(np.arange(256, dtype=np.uint8), (256, 1))
    nb = 16 if elem == 4 else 8
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], nb, 1)
    q = B.MxTensor(torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV), ELEM[elem], nb * 32)
    got = B.dequantize_mx(q, TYPES[out]).cpu()
    want = torch.from_numpy(mx.values(codes, scales, ELEM[elem], nb * 32)).float().to(TYPES[out])
    assert torch.equal(got.isnan(), want.isnan())
    got, want = got.nan_to_num(0, posinf=np.inf, neginf=-np.inf), want.nan_to_num(0, posinf=np.inf, neginf=-np.inf)
    assert torch.equal(got, want)


def test_conversions_leave_what_is_around(B):
    """Results into slices of wider tensors: nothing outside their rows and blocks changes."""
    x = torch.randn(5, 70, device=DEV)
    room = torch.full((7, 128), 99, dtype=torch.uint8, device=DEV)
    sroom = torch.full((7, 12), 77, dtype=torch.uint8, device=DEV)
    q = B.MxTensor(room[1:6, 16:64], sroom[1:6, 4:8], B.MX4, 70)
    B.quantize_mx(x, B.MX4, out=q)
    want = mx.quantize(host(x), B.MX4, mx.COVER)
    same_tensor(q, want, 70)
    assert (host(room[0]) == 99).all() and (host(room[6]) == 99).all() and (host(room[:, :16]) == 99).all() and (host(room[:, 64:]) == 99).all()
    assert (host(sroom[[0, 6]]) == 77).all() and (host(sroom[:, :4]) == 77).all() and (host(sroom[:, 8:]) == 77).all()
    y = torch.full((7, 90), -5.0, device=DEV, dtype=torch.bfloat16)
    B.dequantize_mx(q, torch.bfloat16, out=y[1:6, 3:73])
    assert torch.equal(y[1:6, 3:73].cpu(), torch.from_numpy(mx.values(*want, B.MX4, 70)).bfloat16())
    y[1:6, 3:73] = -5.0
    assert (host(y) == -5).all()


# ---- products ------------------------------------------------------------------------------------ #
def operand(rng, rows, K, elem, spread=6):
    """Codes of every kind (E4M3's NaN codes apart) with scales 2^spread apart at most."""
    nb = -(-K // 32)
    v = rng.standard_normal((rows, K)) * np.exp2(rng.integers(0, spread + 1, (rows, nb)).repeat(32, 1)[:, :K])
    return mx.quantize(v.astype(np.float32), ELEM[elem], mx.COVER)


def on_gpu(B, q, elem, K, garbage=True):
    codes, scales = torch.from_numpy(q[0]).to(DEV), torch.from_numpy(q[1]).to(DEV)
    if garbage:
        scales[:, -(-K // 32):] = 255                      # padding has no effect
    return B.MxTensor(codes, scales, ELEM[elem], K)


def product_bound(x, w, bias, elems, exact):
    """What float32 products and sums of any order are off by, and what the alignment of eight products adds."""
    K = x.shape[1]
    total = np.abs(x) @ np.abs(w).T + (0 if bias is None else np.abs(bias))
    err = (K + 8) * U * total
    if not exact and 8 in elems:
        xp, wp = (torch.nn.functional.pad(torch.from_numpy(np.abs(v)).to(DEV), (0, -K % 8)) for v in (x, w))
        big = sum((xp[:, None, k:k + 8] * wp[None, :, k:k + 8]).amax(2) for k in range(0, K, 8))
        err = err + 7 * 2.0 ** -13 * big.cpu().numpy()
    return err


def products(B, rng, M, N, K, ex, ew, bias):
    qx, qw = operand(rng, M, K, ex), operand(rng, N, K, ew)
    b = rng.standard_normal(N).astype(np.float32) * 8 if bias else None
    x, w = mx.values(*qx, ELEM[ex], K), mx.values(*qw, ELEM[ew], K)
    return (on_gpu(B, qx, ex, K), on_gpu(B, qw, ew, K), None if b is None else torch.from_numpy(b).to(DEV)), (x, w, b)


PAIRS = [(4, 4), (8, 4), (8, 8), (4, 8)]
SHAPES = [(1, 1, 1), (1, 16, 32), (2, 33, 40), (1, 64, 129), (16, 48, 512), (17, 31, 95), (33, 130, 700), (64, 64, 1024), (100, 57, 2999), (129, 200, 256),
          (130, 257, 384), (257, 128, 160)]


@pytest.mark.parametrize("M, N, K", SHAPES)
@pytest.mark.parametrize("ex, ew", PAIRS)
def test_linear(B, ex, ew, M, N, K):
    rng = rng_of(ex, ew, M, N, K)
    (x, w, b), (vx, vw, vb) = products(B, rng, M, N, K, ex, ew, M % 2 == 1)
    bounds = [product_bound(vx, vw, vb, (ex, ew), exact) for exact in (False, True)]
    for relu in (False, True):
        want = mx.linear(vx, vw, vb, relu)
        for out in TYPES:
            y = host(B.linear_mx(x, w, b, relu, TYPES[out]))
            tol = bounds[out == "f32"]
            tol = tol + HALF[out] * (np.abs(want) + tol) + (2.0 ** -25 if out == "f16" else 0)
            ok = np.abs(y - want) <= tol
            ok |= np.isinf(y) & (np.abs(want) + tol > 65504) if out == "f16" else False
            assert ok.all(), (out, relu, np.argwhere(~ok)[:4], np.abs(y - want).max())


def steps_of(v, scale, elem):
    """Half the distance of neighbouring elements around v * 2^-e, in the block's units."""
    table = mx.magnitudes(ELEM[elem])
    a = np.minimum(np.abs(v) / scale, table[-1])
    up = np.clip(np.searchsorted(table, a, side="right"), 1, len(table) - 1)
    return (table[up] - table[up - 1]) / 2 * scale


@pytest.mark.parametrize("M, N, K", [(1, 32, 64), (3, 20, 100), (16, 100, 512), (33, 130, 700), (129, 64, 1024), (130, 257, 384), (300, 288, 256)])
@pytest.mark.parametrize("ex, ew, elem", [(4, 4, 4), (8, 4, 8), (8, 8, 8), (4, 8, 4), (8, 8, 4), (4, 4, 8)])
def test_linear_q(B, ex, ew, elem, M, N, K):
    rng = rng_of(ex, ew, elem, M, N, K)
    (x, w, b), (vx, vw, vb) = products(B, rng, M, N, K, ex, ew, N % 2 == 0)
    err = product_bound(vx, vw, vb, (ex, ew), False)
    for rule, relu in ((mx.COVER, True), (mx.FLOOR, False)):
        q = B.linear_mx_q(x, w, b, ELEM[elem], rule, relu)
        want = mx.linear(vx, vw, vb, relu)
        codes, scales = host(q.codes), host(q.scales)
        nb = -(-N // 32)
        assert not scales[:, nb:].any()
        wide = np.pad(want, ((0, 0), (0, nb * 32 - N)))
        ewide = np.pad(err, ((0, 0), (0, nb * 32 - N)))
        amax, slack = np.abs(wide).reshape(M, nb, 32).max(2), ewide.reshape(M, nb, 32).max(2)
        for m in range(M):
            for k in range(nb):
                lo, hi = (mx.scale_byte(max(a, 0.0), ELEM[elem], rule) for a in (amax[m, k] - slack[m, k], amax[m, k] + slack[m, k]))
                assert lo <= scales[m, k] <= hi
        got = mx.values(codes, scales, ELEM[elem], nb * 32)
        assert not got[:, N:].any() and not (codes == (128 if elem == 8 else 256)).any()
        scale = np.exp2(scales[:, :nb].astype(np.float64) - 127).repeat(32, 1)
        top = mx.magnitudes(ELEM[elem])[-1] * scale
        near = np.clip(wide, -top, top)
        # the largest half step that any value within err of the wanted one meets, and err itself
        half = np.maximum(steps_of(np.abs(near) + ewide, scale, elem), steps_of(near, scale, elem))
        ok = np.abs(got - near) <= ewide + half
        assert ok.all(), (np.argwhere(~ok)[:4], rule)


VARIANT_SHAPES = [(1, 1, 1), (3, 35, 97), (16, 32, 300), (33, 65, 513), (70, 100, 1025), (130, 140, 1600), (257, 300, 700)]


@functools.lru_cache(maxsize=None)
def variant_case(B, ex, ew, M, N, K):
    gpu, (vx, vw, vb) = products(B, rng_of("variant", ex, ew, M, N, K), M, N, K, ex, ew, True)
    return gpu, mx.linear(vx, vw, vb, True), [product_bound(vx, vw, vb, (ex, ew), exact) for exact in (False, True)]


@pytest.mark.parametrize("variant", range(1, 11))
@pytest.mark.parametrize("ex, ew", PAIRS)
def test_linear_by_every_kernel(B, ex, ew, variant):
    """Each kernel on the same calls, tiles of every kind of edge among them: within the bounds, and converted as its own float32 values
    would be (4-bit operands: the same products in every kernel)."""
    for M, N, K in VARIANT_SHAPES:
        (x, w, b), want, bounds = variant_case(B, ex, ew, M, N, K)
        for out in TYPES:
            y = host(B.linear_mx(x, w, b, True, TYPES[out], variant=variant))
            tol = bounds[out == "f32"]
            tol = tol + HALF[out] * (want + tol) + (2.0 ** -25 if out == "f16" else 0)
            ok = (np.abs(y - want) <= tol) | ((out == "f16") & np.isinf(y) & (want + tol > 65504))
            assert ok.all(), (M, N, K, out, np.argwhere(~ok)[:4])
        if variant == 2:                                     # half of a block to a workgroup
            with pytest.raises(B.DfqError):
                B.linear_mx_q(x, w, b, variant=variant)
        else:
            q = B.linear_mx_q(x, w, b, B.MX8, relu=True, variant=variant)
            if ex == ew == 4:
                assert torch.equal(q.codes, B.quantize_mx(B.linear_mx(x, w, b, True, torch.float32, variant=variant)).codes)
            off = np.abs(host(B.dequantize_mx(q)) - want)
            blocks = np.pad(want, ((0, 0), (0, -N % 32))).reshape(M, -1, 32).max(2).repeat(32, 1)[:, :N]
            assert (off <= bounds[0] * (1 + 2.0 ** -3) + np.maximum(2.0 ** -4 * want, 2.0 ** -17 * blocks)).all()


def test_linear_rows_too_far_apart_for_tiles(B):
    """Rows of an operand beyond the reach of 31-bit offsets: by 64-bit addresses, the same sums."""
    rng = rng_of("reach")
    M, N, K, ld = 5, 40, 96, (1 << 22) + 16
    (x, w, b), (vx, vw, vb) = products(B, rng, M, N, K, 8, 4, True)
    room = torch.full((M * ld,), 0x7f, dtype=torch.uint8, device=DEV)
    codes = room.as_strided((M, 96), (ld, 1))
    codes.copy_(x.codes)
    far = B.MxTensor(codes, x.scales, x.elem, K)
    want = mx.linear(vx, vw, vb)
    assert (np.abs(host(B.linear_mx(far, w, b, dtype=torch.float32)) - want) <= product_bound(vx, vw, vb, (8, 4), True) + U * np.abs(want)).all()
    with pytest.raises(B.DfqError):
        B.linear_mx(far, w, b, variant=10)


def test_linear_keeps_what_is_no_number(B):
    """A NaN block, an E4M3 NaN and a scale that overflows reach the outputs that read them, and no others."""
    for ex, ew in PAIRS:
        rng = rng_of("nan", ex, ew)
        (x, w, _), (vx, vw, _) = products(B, rng, 5, 40, 160, ex, ew, False)
        x.scales[1, 2] = 255
        w.scales[7, 4] = 255
        bad = np.zeros((5, 40), bool)
        bad[1], bad[:, 7] = True, True
        if ex == 8:
            x.codes[3, 11] = 0x7f
            bad[3] = True
        if ew == 8:
            w.codes[20, 159] = 0xff
            bad[:, 20] = True
        for out in TYPES:
            assert np.array_equal(np.isnan(host(B.linear_mx(x, w, None, False, TYPES[out]))), bad)
            assert np.array_equal(np.isnan(host(B.linear_mx(x, w, None, True, TYPES[out]))), bad)
        q = B.linear_mx_q(x, w)
        nans = np.isnan(host(B.dequantize_mx(q)))
        blocks = np.stack((bad[:, :32].any(1), bad[:, 32:].any(1)), 1)
        assert np.array_equal(nans, blocks.repeat(32, 1)[:, :40])


@pytest.mark.parametrize("ex, ew", PAIRS)
def test_linear_rows_far_apart(B, ex, ew):
    """Operands and results as slices of wider tensors, rows of the result unaligned: nothing around them changes."""
    M, N, K = 37, 70, 352
    rng = rng_of("far", ex, ew)
    (x, w, b), (vx, vw, vb) = products(B, rng, M, N, K, ex, ew, True)

    def spread(q):
        c = torch.full((q.codes.shape[0] + 2, q.codes.shape[1] + 48), 0x55, dtype=torch.uint8, device=DEV)
        s = torch.full((q.codes.shape[0] + 2, q.scales.shape[1] + 8), 255, dtype=torch.uint8, device=DEV)
        c[1:-1, 16:16 + q.codes.shape[1]] = q.codes
        s[1:-1, 4:4 + q.scales.shape[1]] = q.scales
        return B.MxTensor(c[1:-1, 16:16 + q.codes.shape[1]], s[1:-1, 4:4 + q.scales.shape[1]], q.elem, q.k)

    for out in TYPES:
        room = torch.full((M + 2, N + 5), 3.0, dtype=TYPES[out], device=DEV)
        y = B.linear_mx(spread(x), spread(w), b, False, TYPES[out], out=room[1:-1, 1:N + 1])
        assert torch.equal(y, B.linear_mx(x, w, b, False, TYPES[out]))
        room[1:-1, 1:N + 1] = 3.0
        assert (host(room) == 3).all()
    q = B.MxTensor.empty(M + 2, N + 58, B.MX8, DEV)
    q.codes.fill_(9)
    q.scales.fill_(9)
    part = B.MxTensor(q.codes[1:-1, 32:], q.scales[1:-1, :], B.MX8, N)
    B.linear_mx_q(spread(x), spread(w), b, out=part)
    ref = B.linear_mx_q(x, w, b)
    assert torch.equal(part.codes[:, :96], ref.codes) and torch.equal(part.scales[:, :4], ref.scales)
    assert (host(q.codes[[0, -1]]) == 9).all() and (host(q.codes[:, :32]) == 9).all() and (host(q.scales[[0, -1]]) == 9).all()


def test_linear_one_sum_of_many_equal_terms(B):
    """A long reduction: 16384 products of +1 and one of each sign beside them, exact in every type that holds the count."""
    K = 16384
    for ex, ew in PAIRS:
        one = {4: 2 | 2 << 4, 8: 0x38}
        x = B.MxTensor(torch.full((3, K * ex // 8), one[ex], dtype=torch.uint8, device=DEV), torch.full((3, K // 32), 127, dtype=torch.uint8, device=DEV), ELEM[ex], K)
        w = B.MxTensor(torch.full((50, K * ew // 8), one[ew], dtype=torch.uint8, device=DEV), torch.full((50, K // 32), 127, dtype=torch.uint8, device=DEV), ELEM[ew], K)
        for out in TYPES:
            assert (host(B.linear_mx(x, w, None, False, TYPES[out])) == K).all()


# ---- norm ---------------------------------------------------------------------------------------- #
NORM_U = 64 * U      # at most 64 roundings on the way to a value of the norm (csrc/mx_convert.hip: rows in registers)


@pytest.mark.parametrize("rows, K", [(1, 1), (3, 20), (2, 512), (5, 513), (4, 2048), (3, 3001), (2, 8192), (3, 8225), (2, 32768)])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_rms_norm(B, dtype, rows, K):
    rng = rng_of("norm", dtype, rows, K)
    x, add = (torch.from_numpy(rng.standard_normal((rows, K)) * 3).to(TYPES[dtype]) for _ in range(2))
    weight = torch.from_numpy(1 + 0.3 * rng.standard_normal(K))
    for with_add, wtype, elem, rule in ((True, dtype, 8, mx.COVER), (False, "f32", 4, mx.FLOOR), (True, None, 8, mx.FLOOR), (False, dtype, 4, mx.COVER)):
        w = None if wtype is None else weight.to(TYPES[wtype])
        s, v = mx.rms_norm(x.float().numpy(), add.float().numpy() if with_add else None, None if w is None else host(w), 1e-5)
        q, y, total = B.rms_norm_mx(x.to(DEV), None if w is None else w.to(DEV), 1e-5, add=add.to(DEV) if with_add else None, elem=ELEM[elem], rule=rule,
                                    want_y=True)
        if with_add:
            assert torch.equal(total.cpu(), torch.from_numpy(s).to(TYPES[dtype]))
        else:
            assert total is None
        err = NORM_U * np.abs(v)
        tol = err + HALF[dtype] * (np.abs(v) + err) + (2.0 ** -25 if dtype == "f16" else 0)
        assert (np.abs(host(y) - v) <= tol).all()
        nb = -(-K // 32)
        scales, got = host(q.scales), mx.values(host(q.codes), host(q.scales), ELEM[elem], nb * 32)
        assert not scales[:, nb:].any() and not got[:, K:].any()
        wide = np.pad(v, ((0, 0), (0, nb * 32 - K)))
        amax = np.abs(wide).reshape(rows, nb, 32).max(2)
        for r in range(rows):
            for k in range(nb):
                lo, hi = (mx.scale_byte(amax[r, k] * f, ELEM[elem], rule) for f in (1 - NORM_U, 1 + NORM_U))
                assert lo <= scales[r, k] <= hi
        scale = np.exp2(scales[:, :nb].astype(np.float64) - 127).repeat(32, 1)
        top = mx.magnitudes(ELEM[elem])[-1] * scale
        near = np.clip(wide, -top, top)
        half = np.maximum(steps_of(np.abs(near) * (1 + NORM_U), scale, elem), steps_of(near, scale, elem))
        assert (np.abs(got - near) <= NORM_U * np.abs(wide) + half).all()


@pytest.mark.parametrize("K", [100, 4096, 40000])
def test_rms_norm_in_place_and_strided(B, K):
    """The residual stream updated where it is, from strided and unaligned rows; a row too long for registers among them."""
    rng = rng_of("place", K)
    x, res = (torch.from_numpy(rng.standard_normal((6, K))).to(DEV, torch.bfloat16) for _ in range(2))
    w = torch.from_numpy(1 + 0.1 * rng.standard_normal(K)).to(DEV, torch.bfloat16)
    want = B.rms_norm_mx(x, w, 1e-6, add=res, want_y=True)
    for how in ("dense", "wide", "odd"):
        for onto_x in (False, True):
            xs, rs = strided(x.clone(), how), strided(res.clone(), how)
            q, y, total = B.rms_norm_mx(xs, w, 1e-6, add=rs, want_y=True, sum_out=xs if onto_x else rs)
            assert total is (xs if onto_x else rs) and torch.equal(total, want[2])
            assert torch.equal(q.codes, want[0].codes) and torch.equal(q.scales, want[0].scales) and torch.equal(y, want[1])
            assert torch.equal(rs if onto_x else xs, res if onto_x else x)
    # partly over one another: refused
    room = torch.zeros(7, K, device=DEV, dtype=torch.bfloat16)
    with pytest.raises(B.DfqError):
        B.rms_norm_mx(room[:6], w, 1e-6, add=res, sum_out=room[1:])


def test_rms_norm_rows_that_are_no_numbers(B):
    x = torch.ones(4, 64, device=DEV)
    x[0, 3], x[1, 40], x[2] = float("nan"), float("inf"), 0.0
    q, y, _ = B.rms_norm_mx(x, None, 0.0, want_y=True)
    s = host(q.scales)
    assert (s[0, :2] == 255).all() and s[1, 1] == 255 and s[1, 0] == 0 and (s[2, :2] == 255).all() and (s[3, :2] == s[3, 0]).all() and s[3, 0] != 255
    y = host(y)
    assert np.isnan(y[0]).all() and np.isnan(y[1, 40]) and not y[1, :32].any() and np.isnan(y[2]).all() and (y[3] == 1).all()
    q, y, _ = B.rms_norm_mx(x[2:3], None, 1e-6, want_y=True)
    assert not host(y).any() and not host(q.codes).any() and not host(q.scales).any()


# ---- as they are used ---------------------------------------------------------------------------- #
def block(B, x, res, weight, w1, w2, elem, dtype):
    q, _, total = B.rms_norm_mx(x, weight, 1e-5, add=res)
    return total, B.linear_mx(B.linear_mx_q(q, w1, elem=elem, relu=True), w2, dtype=dtype)


@pytest.mark.parametrize("M", [1, 24, 300])
def test_a_block_of_them(B, M):
    """Norm, product converted for the next, product: every link against the oracle fed with what the link before it gave."""
    d, hidden = 512, 1000
    rng = rng_of("block", M)
    x, res = (torch.from_numpy(rng.standard_normal((M, d))).to(DEV, torch.bfloat16) for _ in range(2))
    weight = torch.ones(d, device=DEV)
    w1, w2 = (B.quantize_mx(torch.from_numpy(rng.standard_normal(s) / s[1] ** 0.5).float().to(DEV), B.MX4) for s in ((hidden, d), (d, hidden)))
    total, y = block(B, x, res, weight, w1, w2, B.MX8, torch.float32)
    q, _, _ = B.rms_norm_mx(x, weight, 1e-5, add=res)
    h = B.linear_mx_q(q, w1, elem=B.MX8, relu=True)
    vh, vw = host(B.dequantize_mx(h)), host(B.dequantize_mx(w2))
    assert (np.abs(host(y) - vh @ vw.T) <= product_bound(vh, vw, None, (8, 4), True) + U * np.abs(vh @ vw.T)).all()
    mid = host(B.linear_mx(q, w1, relu=True, dtype=torch.float32))
    off = np.abs(vh - mid).max() / np.abs(mid).max()
    assert off <= 2.0 ** -4 + 2.0 ** -9          # half a step of E4M3 beside a block's largest
    assert torch.equal(total, (x.float() + res.float()).bfloat16())


def test_captured_and_replayed(B):
    """The block in a graph, replayed on new inputs between eager work."""
    d, hidden, M = 256, 384, 20
    rng = rng_of("graph")
    fresh = lambda: torch.from_numpy(rng.standard_normal((M, d))).to(DEV, torch.bfloat16)
    x, res = fresh(), fresh()
    weight = torch.ones(d, device=DEV, dtype=torch.bfloat16)
    w1, w2 = (B.quantize_mx(torch.from_numpy(rng.standard_normal(s)).float().to(DEV), e) for s, e in (((hidden, d), B.MX4), ((d, hidden), B.MX8)))
    run = lambda a, r: block(B, a, r, weight, w1, w2, B.MX4, torch.bfloat16)
    run(x, res)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(x, res)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        total, y = run(x, res)
    for _ in range(3):
        x.copy_(fresh())
        res.copy_(fresh())
        graph.replay()
        torch.cuda.synchronize()
        t, z = run(x, res)
        assert torch.equal(t, total) and torch.equal(z, y)


def test_on_a_stream_of_its_own(B):
    side = torch.cuda.Stream()
    x = torch.randn(64, 320, device=DEV)
    want = B.linear_mx(B.quantize_mx(x), B.quantize_mx(x, B.MX4))
    side.wait_stream(torch.cuda.current_stream())
    for s in (side, side.cuda_stream):
        got = B.linear_mx(B.quantize_mx(x, stream=s), B.quantize_mx(x, B.MX4, stream=s), stream=s)
        side.synchronize()
        assert torch.equal(got, want)


def test_tensors_of_more_dimensions_and_refusals(B):
    x = torch.randn(2, 3, 96, device=DEV)
    q = B.quantize_mx(x)
    assert q.codes.shape == (6, 96) and torch.equal(q.codes, B.quantize_mx(x.view(6, 96)).codes)
    q2, y, total = B.rms_norm_mx(x, add=x, want_y=True)
    assert y.shape == x.shape and total.shape == x.shape and q2.codes.shape == (6, 96)
    w = B.quantize_mx(torch.randn(40, 96, device=DEV), B.MX4)
    bad = [lambda: B.quantize_mx(x.transpose(0, 1)), lambda: B.quantize_mx(x[0].t()), lambda: B.quantize_mx(x[0, :1].expand(4, 96)),
           lambda: B.linear_mx(q, w._replace(k=64)), lambda: B.linear_mx(q, w, torch.zeros(39, device=DEV)), lambda: B.linear_mx(q, w, out=torch.zeros(6, 41, device=DEV), dtype=torch.float32),
           lambda: B.linear_mx(q._replace(codes=q.codes[:5]), w), lambda: B.linear_mx(q, w._replace(elem=B.MX8)), lambda: B.dequantize_mx(q._replace(k=0)),
           lambda: B.quantize_mx(x, out=q._replace(elem=B.MX4)), lambda: B.linear_mx_q(q, w, out=B.MxTensor.empty(6, 39, B.MX8)), lambda: B.rms_norm_mx(x, add=x[0]),
           lambda: B.rms_norm_mx(x, weight=torch.ones(95, device=DEV))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: B.quantize_mx(x.double()), lambda: B.quantize_mx(x.int()), lambda: B.rms_norm_mx(x, add=x.bfloat16())):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: B.quantize_mx(x, rule=3), lambda: B.rms_norm_mx(x, eps=-1.0), lambda: B.rms_norm_mx(x, elem=None), lambda: B.quantize_mx(x, out=B.MxTensor(x.view(torch.uint8).view(6, -1), q.scales, B.MX8, 96))):
        with pytest.raises(B.DfqError):
            call()
    empty = B.quantize_mx(x[:0].view(0, 96))
    assert B.linear_mx(empty, w).shape == (0, 40) and B.dequantize_mx(empty).shape == (0, 96) and B.linear_mx_q(empty, w).codes.shape == (0, 64)
    assert B.rms_norm_mx(x[:0].view(0, 96))[0].codes.shape == (0, 96)


def test_norm_of_more_rows_than_one_grid_holds(B):
    """2^28 + 37 rows of one value, 16 threads to a row: the threads no longer fit 32 bits.  x / |x| of +-2 is exact."""
    rows = (1 << 28) + 37
    x = (torch.randint(0, 2, (rows, 1), device=DEV, dtype=torch.int8) * 4 - 2).bfloat16()
    q, y, _ = B.rms_norm_mx(x, eps=0.0, elem=B.MX4, want_y=True)
    assert torch.equal(y, x * 0.5)
    want = B.quantize_mx(torch.tensor([[1.0], [-1.0]], device=DEV), B.MX4)
    for first in range(0, rows, 1 << 26):
        part = slice(first, first + (1 << 26))
        negative = x[part] < 0
        assert torch.equal(q.codes[part, :1], torch.where(negative, want.codes[1, 0], want.codes[0, 0])) and not q.codes[part, 1:].any()
        assert torch.equal(q.scales[part, 0], want.scales[0, 0].expand(negative.shape[0])) and not q.scales[part, 1:].any()


@pytest.mark.parametrize("variant", [2, 6, 10])
def test_linear_of_more_tokens_than_one_grid_holds(B, variant):
    """2^30 + 5 tokens: 2^24 tiles of 256 threads and more.  The first value of each token times 1."""
    M = (1 << 30) + 5
    x = B.MxTensor(torch.randint(0, 256, (M, 16), device=DEV, dtype=torch.uint8), torch.full((M, 4), 128, device=DEV, dtype=torch.uint8), B.MX4, 32)
    w = B.quantize_mx(torch.eye(1, 32, device=DEV), B.MX4)
    y = torch.full((M, 1), 77.0, device=DEV, dtype=torch.bfloat16)
    B.linear_mx(x, w, out=y, dtype=torch.bfloat16, variant=variant)
    magnitude = mx.magnitudes(mx.MX4)
    table = torch.tensor(np.concatenate((magnitude, -magnitude)) * 2, device=DEV, dtype=torch.bfloat16)
    step = 1 << 26
    for first in range(0, M, step):
        assert torch.equal(y[first:first + step, 0], table[(x.codes[first:first + step, 0] & 15).int()])


@pytest.mark.parametrize("K", [1, 20, 512, 3001, 8192, 16384, 40000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rms_norm_of_rows_whose_squares_leave_the_range(B, dtype, K):
    """Rows from float32's smallest values to its largest ones, several of them to a wavefront; 1e-30 and 0 for eps."""
    rng = rng_of("range", dtype, K)
    powers = (-146, -130, -126, -100, -64, -45, -41, -40, -39, 0, 40, 49, 50, 51, 64, 100, 120, 126)
    x = torch.from_numpy(np.clip(rng.standard_normal((len(powers), K)), -1.9, 1.9) * np.exp2(np.array(powers, np.float64))[:, None]).to(TYPES[dtype])
    x[:, 0] = torch.from_numpy(np.exp2(np.array(powers, np.float64))).to(TYPES[dtype])      # (a row of zeros: 2^-146 in bfloat16, NaN with eps = 0)
    for eps in (0.0, 1e-30):
        with np.errstate(invalid="ignore"):
            _, v = mx.rms_norm(x.float().numpy(), None, None, eps)
        q, y, _ = B.rms_norm_mx(x.to(DEV), None, eps, want_y=True)
        err = NORM_U * np.abs(v)
        tol = err + HALF[dtype] * (np.abs(v) + err) + 2.0 ** (-150 if dtype == "f32" else -134)
        assert ((np.abs(host(y) - v) <= tol) | np.isnan(host(y)) & np.isnan(v)).all()
        same = B.quantize_mx(y.float())
        if dtype == "f32":
            assert torch.equal(q.codes, same.codes) and torch.equal(q.scales, same.scales)


def test_tensors_of_more_than_four_gigabytes(B):
    """Rows behind 2^32 bytes and 2^32 values of a tensor are converted, converted back and multiplied like the same rows alone."""
    rows, K = (1 << 22) + 3, 1100
    x = torch.empty(rows, K, device=DEV, dtype=torch.bfloat16)
    x.view(-1)[:] = 0.5
    some = torch.randn(70, K, device=DEV).bfloat16()
    x[-70:] = some
    q, alone = B.quantize_mx(x, B.MX8), B.quantize_mx(some, B.MX8)
    assert torch.equal(q.codes[-70:], alone.codes) and torch.equal(q.scales[-70:], alone.scales)
    assert torch.equal(q.codes[:70], q.codes[rows // 2:rows // 2 + 70])
    assert torch.equal(B.dequantize_mx(q, torch.bfloat16, out=x)[-70:], B.dequantize_mx(alone, torch.bfloat16))
    few = B.quantize_mx(torch.randn(3, K, device=DEV), B.MX4)
    weights = lambda t, n: B.MxTensor(t.codes[:n], t.scales[:n], t.elem, t.k)
    last = B.MxTensor(q.codes[-(1 << 22):], q.scales[-(1 << 22):], q.elem, q.k)             # as weights: 2^22 features
    for variant in (2, 5, 6, 10):
        y = B.linear_mx(few, last, variant=variant)
        assert torch.equal(y[:, -70:], B.linear_mx(few, alone, variant=variant)), variant
        assert torch.equal(y[:, :32], B.linear_mx(few, weights(last, 32), variant=variant)), variant


def test_one_tensor_as_both_operands_and_rows_of_a_padded_batch(B):
    """x times itself; rows that hold no numbers leave the others as they are."""
    x = torch.randn(300, 260, device=DEV)
    for elem in (B.MX4, B.MX8):
        q = B.quantize_mx(x, elem)
        copy = q._replace(codes=q.codes.clone(), scales=q.scales.clone())
        want = B.linear_mx(q, copy, dtype=torch.float32)
        assert torch.equal(B.linear_mx(q, q, dtype=torch.float32), want)
        padded = copy._replace(codes=copy.codes.clone(), scales=copy.scales.clone())
        padded.codes[100:150], padded.scales[100:150] = 0xff, 0xff
        for variant in range(1, 11):
            y, z = (B.linear_mx(t, q, dtype=torch.float32, variant=variant) for t in (copy, padded))
            assert torch.equal(z[:100], y[:100]) and torch.equal(z[150:], y[150:]) and torch.isnan(z[100:150]).all(), variant


def test_calls_from_two_threads(B):
    import threading
    x, w = B.quantize_mx(torch.randn(40, 500, device=DEV)), B.quantize_mx(torch.randn(130, 500, device=DEV), B.MX4)
    h = torch.randn(40, 500, device=DEV, dtype=torch.bfloat16)
    want = [B.linear_mx(x, w), B.linear_mx_q(x, w).codes, B.rms_norm_mx(h)[0].codes, B.quantize_mx(h).codes]
    torch.cuda.synchronize()
    wrong = []

    def work(stream):
        with torch.cuda.stream(stream):
            for _ in range(50):
                got = [B.linear_mx(x, w), B.linear_mx_q(x, w).codes, B.rms_norm_mx(h)[0].codes, B.quantize_mx(h).codes]
                stream.synchronize()
                wrong.extend(i for i, (a, b) in enumerate(zip(got, want)) if not torch.equal(a, b))

    threads = [threading.Thread(target=work, args=(torch.cuda.Stream(),)) for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
