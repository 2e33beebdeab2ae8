"""The microscaled messages (adpsgd_mx_*) on the GPU against the 64-bit reference in mx_reference.py.

Tolerances, from the arithmetic:
- quantize: bit-equal.  Each sum is one fp32 rounding on both sides, the scale and the rounding are exact.
- dequantize: one fp32 addition, bit-equal.
- average: the mean is a 64-bit sum of numbers of at most four significant bits; base + mean is rounded
  once to fp32: half a step, 2^-24 of the value.  Variances: 64-bit sums of non-negative terms, 1e-12.
- product: a wave sums at most 16384 products in fp32, by instructions of at least 32 products and at
  most four roundings each (2^-24 of the magnitudes' sum apiece); then one rounding for the partial sum
  and one for the result.
"""
import sys

import numpy as np
import pytest
import torch

import mx_reference as ref

pytestmark = pytest.mark.gpu

FORMATS = [ref.E2M1, ref.E4M3]


@pytest.fixture(scope="module")
def A():
    assert torch.cuda.is_available()
    import paper_2007_06134_amd as A
    return A


def _say(msg):
    print(msg, file=sys.stderr, flush=True)


def _bits(a):
    return np.ascontiguousarray(a, dtype=np.float32).view(np.int32)


def _same(got, want):
    """Equal bits, any NaN equal to any other."""
    got, want = np.asarray(got, dtype=np.float32), np.asarray(want, dtype=np.float32)
    nan = np.isnan(want)
    off = np.argwhere((np.isnan(got) != nan) | (~nan & (_bits(got) != _bits(want))))
    for at in off[:4]:
        _say(f"  at {tuple(at)} of {want.shape}: {got[tuple(at)]!r}, not {want[tuple(at)]!r} ({len(off)} in all)")
    return len(off) == 0


def _device_rows(a, layout, fill=7.5):
    """a [K, P] float32 on the device: rows padded, packed, or packed and one element off a 16-byte
    boundary; the memory around the rows holds `fill`.  Returns (view, whole buffer)."""
    K, P = a.shape
    ld = P if layout != "padded" else -(-P // 256) * 256 + 256
    lead = 1 if layout == "off" else 0
    buf = torch.full((lead + K * ld + 64,), fill, device="cuda")
    view = torch.as_strided(buf, (K, P), (ld, 1), lead)
    view.copy_(torch.from_numpy(a))
    return view, buf


def _outside_untouched(view, buf, fill=7.5):
    keep = torch.ones_like(buf, dtype=torch.bool)
    torch.as_strided(keep, view.shape, view.stride(), view.storage_offset()).fill_(False)
    return bool((buf[keep] == fill).all())


def _numbers(rng, K, P, spread=True):
    """Normal numbers whose size changes from stretch to stretch, zero stretches among them."""
    a = rng.standard_normal((K, P))
    if spread:
        a *= np.repeat(10.0 ** rng.uniform(-6, 2, P // 40 + 1), 40)[:P]
        a[:, rng.integers(0, P):][:, :50] = 0.0
    return a.astype(np.float32)


def _message(rng, K, P, fmt):
    """(codes uint8 [K, bytes], scale bytes [K, blocks], values) of a message of ordinary numbers."""
    c, byte, v = ref.quantize(_numbers(rng, K, P), fmt)
    return ref.pack(c, fmt), byte.astype(np.uint8), v


def _rows(A, codes, byte, P, fmt, pad=True):
    """MxRows of host bytes; the bytes past a row's end are 0xEE."""
    def put(a):
        w = a.shape[1] + (16 - a.shape[1]) % 16 + (32 if pad else 0)
        t = torch.full((a.shape[0], w), 0xEE, dtype=torch.uint8)
        t[:, :a.shape[1]] = torch.from_numpy(np.ascontiguousarray(a))
        return t.cuda()
    return A.MxRows(put(codes), put(byte), P, fmt)


SHAPES = [(1, 1), (1, 31), (2, 32), (3, 33), (1, 255), (2, 1024), (3, 1025), (5, 4099), (33, 2000), (4, 65_536),
          (100, 777), (3, 2_100_003)]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("K,P", SHAPES)
@pytest.mark.parametrize("layout,with_base,with_res", [("padded", True, True), ("packed", False, True),
                                                       ("off", True, False), ("off", False, False)])
def test_quantize_bits(A, fmt, K, P, layout, with_base, with_res):
    _say(f"quantize {fmt} K={K} P={P} {layout} base={with_base} residual={with_res}")
    rng = np.random.default_rng([fmt, K, P])
    x = _numbers(rng, K, P)
    base = _numbers(rng, 1, P)[0] if with_base else None
    res = (0.1 * _numbers(rng, K, P)).astype(np.float32) if with_res else None
    if with_base:
        x = (x + base).astype(np.float32)
    d = ref.difference(x, base, res)
    c, byte, v = ref.quantize(d, fmt)
    xd, xbuf = _device_rows(x, layout)
    rd = rbuf = None
    if with_res:
        rd, rbuf = _device_rows(res, layout)
    out_r, out_buf = _device_rows(np.zeros((K, P), np.float32), layout)
    rows = A.MxRows.empty(K, P, fmt)
    rows.codes.fill_(0xEE)
    rows.scales.fill_(0xEE)
    A.mx_quantize(xd, None if base is None else torch.from_numpy(base).cuda(), rd, residual_out=out_r, out=rows)
    torch.cuda.synchronize()
    want = ref.pack(c, fmt)
    assert np.array_equal(rows.codes.cpu().numpy()[:, :want.shape[1]], want)
    assert np.array_equal(rows.scales.cpu().numpy()[:, :byte.shape[1]], byte)
    assert bool((rows.codes[:, want.shape[1]:] == 0xEE).all()) and bool((rows.scales[:, byte.shape[1]:] == 0xEE).all())
    assert _same(out_r.cpu().numpy(), (d.astype(np.float64) - v))
    assert _outside_untouched(out_r, out_buf) and _outside_untouched(xd, xbuf)
    if with_res:     # in place gives the same
        assert _same(rd.cpu().numpy(), res)
        A.mx_quantize(xd, None if base is None else torch.from_numpy(base).cuda(), rd, out=rows)
        assert torch.equal(rd, out_r) and _outside_untouched(rd, rbuf)


@pytest.mark.parametrize("fmt", FORMATS)
def test_quantize_special_blocks(A, fmt):
    """Blocks of zeros, ties, the largest and the least numbers, and blocks that hold NaN or infinities."""
    g = ref.grid(fmt)[:8 if fmt == ref.E2M1 else 127]
    mid = (g[1:] + g[:-1]) / 2
    rng = np.random.default_rng(5)
    blocks = [np.zeros(32), -np.zeros(32)]
    for s in (1.0, 2.0 ** -100, 2.0 ** 60):
        t = np.concatenate([mid, -mid, np.nextafter(mid.astype(np.float32), np.float32(9e9))])
        for i in range(0, len(t), 31):
            part = t[i:i + 31]
            blocks.append(s * np.concatenate([[g[-1]], part, np.zeros(31 - len(part))]))
    tiny = 2.0 ** -149
    for top in (tiny, 3 * tiny, 2.0 ** -127, 2.0 ** -126, 1.75 * 2.0 ** -126, 2.0 ** -125, 2.0 ** -118, 3.4e38,
                1.5 * 2.0 ** 127, 1.75 * 2.0 ** 127, np.nextafter(np.float32(1.5), np.float32(2)) * 2.0 ** 100):
        blocks.append(np.concatenate([[top], rng.uniform(-top, top, 31)]))
    for bad in (np.nan, np.inf, -np.inf):
        for at in (0, 13, 31):
            b = rng.standard_normal(32)
            b[at] = bad
            blocks.append(b)
    blocks.append(rng.standard_normal(32))
    x = np.concatenate(blocks).astype(np.float32)[None]
    c, byte, v = ref.quantize(x, fmt)
    rows = A.MxRows.empty(1, x.shape[1], fmt)
    res = torch.full((1, x.shape[1]), 9.0, device="cuda")
    A.mx_quantize(torch.from_numpy(x).cuda(), residual_out=res, out=rows)
    want = ref.pack(c, fmt)
    ok = np.repeat(byte[0] != 255, 16 if fmt == ref.E2M1 else 32)
    assert np.array_equal(rows.codes.cpu().numpy()[0, :want.shape[1]][ok], want[0][ok])
    assert np.array_equal(rows.scales.cpu().numpy()[0, :byte.shape[1]], byte[0])
    assert (byte == 255).sum() == 9
    with np.errstate(invalid="ignore"):
        assert _same(res.cpu().numpy(), np.where(np.isnan(v), 0.0, x.astype(np.float64) - v))
    assert _same(A.mx_dequantize(rows).cpu().numpy(), v)


@pytest.mark.parametrize("fmt", FORMATS)
def test_dequantize_every_code_and_scale(A, fmt):
    """All codes under all scale bytes, as any sender may have written them."""
    codes = np.arange(256, dtype=np.uint8)
    per = 16 if fmt == ref.E2M1 else 32
    row = np.concatenate([codes, codes])[:512]
    n = 512 // per
    K = 256
    byte = np.repeat(np.arange(256, dtype=np.uint8)[:, None], n, 1)
    P = n * 32 - 5
    rows = _rows(A, np.repeat(row[None], K, 0), byte, P, fmt)
    v = ref.values(np.repeat(row[None], K, 0), byte, P, fmt)
    with np.errstate(over="ignore"):
        want = v.astype(np.float32)      # (6 * 2^127 is an infinity)
    assert _same(A.mx_dequantize(rows).cpu().numpy(), want)
    base = np.random.default_rng(0).standard_normal(P).astype(np.float32)
    with np.errstate(over="ignore"):
        want = (base + want).astype(np.float32)
    assert _same(A.mx_dequantize(rows, torch.from_numpy(base).cuda()).cpu().numpy(), want)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("K,P", SHAPES)
@pytest.mark.parametrize("layout", ["padded", "off"])
def test_dequantize_bits(A, fmt, K, P, layout):
    _say(f"dequantize {fmt} K={K} P={P} {layout}")
    rng = np.random.default_rng([fmt, K, P, 1])
    codes, byte, v = _message(rng, K, P, fmt)
    rows = _rows(A, codes, byte, P, fmt, pad=layout == "padded")
    base = rng.standard_normal(P).astype(np.float32)
    y, buf = _device_rows(np.zeros((K, P), np.float32), layout)
    A.mx_dequantize(rows, torch.from_numpy(base).cuda(), out=y)
    assert _same(y.cpu().numpy(), base + v.astype(np.float32)) and _outside_untouched(y, buf)
    A.mx_dequantize(rows, out=y)
    assert _same(y.cpu().numpy(), v) and _outside_untouched(y, buf)


def _cuts(rng, P, kind):
    """Tensor boundaries: one tensor; empty ones at both ends and between; ones; block and chunk edges."""
    if kind == "one":
        return np.array([0, P])
    if kind == "empty":
        m = sorted(rng.integers(0, P + 1, 3).tolist())
        return np.array([0, 0, 0] + m + [m[-1], P, P, P])
    if kind == "ones":
        n = min(P, 1500)
        return np.array(list(range(n)) + [P])
    if kind == "singles":  # more tensors than two steps of 64 tell apart
        return np.arange(P + 1)
    if kind == "edges":
        marks = [v + d for v in (32, 256, 512, 1024, 2048, 4096, 8192, 16384) for d in (-1, 0, 1) if v + d < P]
        return np.array([0] + sorted(marks) + [P])
    if kind == "gaps":     # runs of empty tensors, longer than a wave's 64, at edges and anywhere
        at = [0, 1, 1024, 1024, 2048, P - 1, P] + rng.integers(0, P + 1, 9).tolist()
        return np.array([0] + sorted(v for a in at for v in [a] * int(rng.integers(1, 300))) + [P])
    n = int(min(P, 400))
    return np.array([0] + sorted(rng.integers(0, P + 1, n).tolist()) + [P])


AVERAGE = [(1, 1, "one"), (2, 31, "empty"), (3, 33, "ones"), (8, 1025, "edges"), (5, 4099, "edges"), (16, 20_000, "many"),
           (33, 2000, "ones"), (100, 777, "many"), (3, 70_000, "empty"), (2, 4_300_007, "many"), (3, 4_200_000, "one"),
           (7, 4_250_001, "edges"), (4, 5000, "gaps"), (3, 4_200_000, "gaps"), (2, 20_000, "singles")]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("K,P,cuts", AVERAGE)
@pytest.mark.parametrize("layout", ["padded", "off"])
def test_average(A, fmt, K, P, cuts, layout):
    _say(f"average {fmt} K={K} P={P} {cuts} {layout}")
    rng = np.random.default_rng([fmt, K, P, 2])
    codes, byte, v = _message(rng, K, P, fmt)
    off = _cuts(rng, P, cuts)
    base = rng.standard_normal(P).astype(np.float32)
    rows = _rows(A, codes, byte, P, fmt)
    offd = torch.from_numpy(off).cuda()
    for b in (base, None):
        new, var = ref.average(v, off, b)
        x, buf = _device_rows(np.zeros((K, P), np.float32), layout)
        got, got_var = A.mx_average(rows, offd, None if b is None else torch.from_numpy(b).cuda(), x=x)
        got, got_var = got.cpu().numpy().astype(np.float64), got_var.cpu().numpy()
        assert np.all(np.abs(got - new) <= 2.0 ** -24 * (1 + 1e-6) * np.abs(new) + 2.0 ** -149)
        assert np.all(np.abs(got_var - var) <= 1e-12 * var)
        assert _same(x.cpu().numpy(), np.repeat(got[None], K, 0)) and _outside_untouched(x, buf)
    # without x, and in place: the same model and variances, bit for bit
    bd = torch.from_numpy(base).cuda()
    first, var1 = A.mx_average(rows, offd, bd)
    again, var2 = A.mx_average(rows, offd, bd, base_out=bd)
    assert again is bd and torch.equal(first, bd) and torch.equal(var1, var2)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("K", [2, 3, 8, 100])
def test_average_of_equal_messages_has_no_variance(A, fmt, K):
    P = 5000
    rng = np.random.default_rng(K)
    codes, byte, v = _message(rng, 1, P, fmt)
    rows = _rows(A, np.repeat(codes, K, 0), np.repeat(byte, K, 0), P, fmt)
    off = torch.tensor([0, 100, 100, 4097, P], device="cuda")
    new, var = A.mx_average(rows, off)
    # (as numbers: a sum of zeros, whatever their signs, is +0)
    assert np.array_equal(new.cpu().numpy().astype(np.float64), v[0]) and bool((var == 0).all())


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_bad_block_reaches_its_own_tensors_only(A, fmt):
    """A block of one worker that could not be sent: NaN in that block's elements of the model, in the
    variance of the tensors that own elements of it, and in that worker's inner products there."""
    K, P = 4, 9000
    rng = np.random.default_rng(3)
    codes, byte, v = _message(rng, K, P, fmt)
    byte[2, 100] = 255                                   # elements 3200 .. 3231
    v = ref.values(codes, byte, P, fmt)
    off = np.array([0, 1000, 3200, 3210, 3232, 3232, 3300, P])
    hit = np.array([False, False, True, True, False, False, False])
    rows, offd = _rows(A, codes, byte, P, fmt), torch.from_numpy(off).cuda()
    new, var = A.mx_average(rows, offd)
    assert np.array_equal(np.isnan(new.cpu().numpy()), np.isnan(v).any(0))
    assert np.array_equal(np.isnan(var.cpu().numpy()), hit)
    c = A.mx_product(rows, offd).cpu().numpy()
    want = np.zeros((7, K, K), bool)
    want[hit, 2, :] = want[hit, :, 2] = True
    assert np.array_equal(np.isnan(c), want)
    # the same as two sets of messages: only the first's row
    c = A.mx_product(rows, offd, _rows(A, codes, np.where(byte == 255, 120, byte).astype(np.uint8), P, fmt)).cpu().numpy()
    want[:] = False
    want[hit, 2, :] = True
    assert np.array_equal(np.isnan(c), want)


def _product_tol(off, mag):
    n = np.diff(off).clip(0, 16384)
    return ((4 * np.ceil(n / 32) + 8) * 2.0 ** -24)[:, None, None] * mag + 1e-37


PRODUCT = [(1, 1, "one"), (2, 31, "empty"), (3, 33, "ones"), (8, 1025, "edges"), (16, 4099, "edges"), (17, 20_000, "many"),
           (32, 9000, "many"), (33, 2000, "ones"), (48, 30_000, "many"), (49, 3000, "many"), (64, 3000, "edges"), (65, 2500, "many"),
           (96, 20_000, "edges"), (130, 1500, "empty"), (100, 777, "many"),
           (256, 600, "empty"), (80, 40_000, "many"), (256, 9000, "edges"), (4, 70_000, "empty"), (8, 300_007, "one"), (2, 4_300_007, "many"), (5, 2_000_000, "one"),
           (4, 5000, "gaps"), (20, 40_000, "gaps"), (40, 5000, "gaps"),
           # stretches that share a tile
           (1, 4_400_000, "edges"), (3, 1_100_000, "many"), (4, 1_050_000, "gaps"), (7, 700_003, "many"), (8, 600_000, "edges"),
           (2, 20_000, "singles"), (17, 10_000, "singles")]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("K,P,cuts", PRODUCT)
def test_product(A, fmt, K, P, cuts):
    _say(f"product {fmt} K={K} P={P} {cuts}")
    rng = np.random.default_rng([fmt, K, P, 4])
    codes, byte, v = _message(rng, K, P, fmt)
    off = _cuts(rng, P, cuts)
    if len(off) * K * K > 20_000_000:
        off = off[:: len(off) * K * K // 20_000_000 + 1]
        off[-1] = P
    rows, offd = _rows(A, codes, byte, P, fmt), torch.from_numpy(off).cuda()
    want, mag = ref.product(v, v, off)
    got = A.mx_product(rows, offd).cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - want) <= _product_tol(off, mag))
    assert np.array_equal(got, got.transpose(0, 2, 1))
    assert np.array_equal(got, A.mx_product(rows, offd, rows).cpu().numpy())
    codes2, byte2, w = _message(rng, K, P, fmt)
    want, mag = ref.product(v, w, off)
    other = _rows(A, codes2, byte2, P, fmt, pad=False)
    got = A.mx_product(rows, offd, other).cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - want) <= _product_tol(off, mag))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("K", [66, 97])
def test_product_of_many_workers_and_long_rows(A, fmt, K):
    """Against 64-bit products of what mx_dequantize reads, itself tested for every code and scale."""
    P = (1 << 22) + 77
    _say(f"product {fmt} K={K} P={P}")
    torch.manual_seed(K)
    x = torch.randn((K, P), device="cuda")
    rows = A.mx_quantize(x, format=fmt)
    v = A.mx_dequantize(rows, out=x)
    off = np.array([0, 1, 5000, 5000, 70_001, 2_500_000, P - 3, P])
    got = A.mx_product(rows, torch.from_numpy(off).cuda()).cpu().numpy().astype(np.float64)
    for t, (lo, hi) in enumerate(zip(off[:-1], off[1:])):
        want, mag = torch.zeros((2, K, K), dtype=torch.float64, device="cuda")
        for at in range(lo, hi, 1 << 19):
            d = v[:, at:min(at + (1 << 19), hi)].double()
            want += d @ d.t().contiguous()
            mag += d.abs() @ d.abs().t().contiguous()
        tol = _product_tol(np.array([lo, hi]), mag.cpu().numpy()[None])[0]
        assert np.all(np.abs(got[t] - want.cpu().numpy()) <= tol)
    assert np.array_equal(got, got.transpose(0, 2, 1))


@pytest.mark.parametrize("K", [5, 16, 40, 70])
def test_eight_bit_products_are_summed_in_two_levels(A, K):
    """Positive elements, whose partial sums only grow: 8 matrix instructions a level of 256 elements, then
    at most 64 of those sums, the joins in 64 bits and the result's rounding."""
    P = 600_000
    torch.manual_seed(K)
    x = torch.rand((K, P), device="cuda") + 0.1
    rows = A.mx_quantize(x, format=A.MX_E4M3)
    v = A.mx_dequantize(rows).double()
    got = A.mx_product(rows, torch.tensor([0, P], device="cuda"))[0].double()
    want = v @ v.t().contiguous()
    assert bool(((got - want).abs() <= (4 * 8 + 64 + 2) * 2.0 ** -24 * want).all())


@pytest.mark.parametrize("K", [1, 3, 8, 16, 20, 40, 60, 70])
def test_product_of_four_bit_messages_of_one_scale_is_exact(A, K):
    """E2M1 products are quarters of integers up to 144: sums of 16384 of them fit an fp32 mantissa."""
    P = 16_384
    rng = np.random.default_rng(K)
    codes = rng.integers(0, 256, (K, P // 2), dtype=np.uint8)
    byte = np.full((K, P // 32), 127, np.uint8)
    v = ref.values(codes, byte, P, ref.E2M1)
    rows = _rows(A, codes, byte, P, ref.E2M1)
    off = np.array([0, 1, 40, 5000, 5003, P])
    got = A.mx_product(rows, torch.from_numpy(off).cuda()).cpu().numpy()
    assert np.array_equal(got.astype(np.float64), ref.product(v, v, off)[0])


@pytest.mark.parametrize("fmt", FORMATS)
def test_product_of_far_scales(A, fmt):
    """Rows of very large and very small numbers: their inner products are those of their scales, as far
    as fp32 reaches (8-bit elements below 2^-126 are rounded to bf16's multiples of 2^-133)."""
    P = 600
    rng = np.random.default_rng(8)
    bytes_ = np.array([0, 1, 20, 127, 190, 230])          # 2^-127 ... 2^103
    codes, _, _ = _message(rng, 6, P, fmt)
    byte = np.repeat(bytes_[:, None], -(-P // 32), 1).astype(np.uint8)
    v = ref.values(codes, byte, P, fmt)
    if fmt == ref.E4M3:
        v = np.where(np.abs(v) < 2.0 ** -126, np.round(v * 2.0 ** 133) * 2.0 ** -133, v)
    off = np.array([0, 100, P])
    want, mag = ref.product(v, v, off)
    got = A.mx_product(_rows(A, codes, byte, P, fmt), torch.from_numpy(off).cuda()).cpu().numpy().astype(np.float64)
    fits = (mag < 2.0 ** 127) & (mag > 2.0 ** -100)       # no sum passes fp32, no product of weight is subnormal
    assert fits.sum() > 20
    # (a product below 2^-126 may be dropped: P of them)
    off_by = (np.abs(got - want) - _product_tol(off, mag) - P * 2.0 ** -126)
    _say(f"  past the tolerance: {[(tuple(i), got[tuple(i)], want[tuple(i)]) for i in np.argwhere((off_by > 0) & fits)[:6]]}")
    assert np.all((off_by <= 0)[fits])
    # products past fp32 are infinities, and of both signs their sum is NaN
    assert not np.any(np.isfinite(got[mag > 2.0 ** 140]))


@pytest.mark.parametrize("fmt", FORMATS)
def test_product_gives_the_averages_variance(A, fmt):
    """(tr C - 1'C1 / K) / K of the inner products is the variance that mx_average gives."""
    K, P = 8, 50_000
    rng = np.random.default_rng(9)
    codes, byte, _ = _message(rng, K, P, fmt)
    rows = _rows(A, codes, byte, P, fmt)
    off = torch.tensor([0, 3, 1000, 1000, 40_001, P], device="cuda")
    _, var = A.mx_average(rows, off)
    c = A.mx_product(rows, off).double()
    tr = c.diagonal(dim1=1, dim2=2).sum(1)
    got = (tr - c.sum((1, 2)) / K) / K
    # fp32 products: (4 n / 32 + 8) 2^-24 of tr at most for each of the K + K^2 sums' weight
    assert bool(((got - var).abs() <= (4 * 16384 / 32 + 8) * 2.0 ** -24 * 2 * tr / K).all())


@pytest.mark.parametrize("fmt", FORMATS)
def test_no_parameters(A, fmt):
    """P = 0: nothing to send, variances and inner products of nothing."""
    rows = A.MxRows(torch.empty((3, 0), dtype=torch.uint8, device="cuda"),
                    torch.empty((3, 0), dtype=torch.uint8, device="cuda"), 0, fmt)
    A.mx_quantize(torch.empty((3, 0), device="cuda"), out=rows)
    assert A.mx_dequantize(rows).shape == (3, 0)
    off = torch.zeros(3, dtype=torch.int64, device="cuda")
    new, var = A.mx_average(rows, off)
    assert new.shape == (0,) and var.tolist() == [0.0, 0.0]
    assert A.mx_product(rows, off).abs().max().item() == 0


def test_as_many_tensors_as_a_call_takes(A):
    """2^24 tensors, of one element each but the last: every kernel's grid still fits a launch."""
    K, T = 2, 1 << 24
    P = T + 1000
    torch.manual_seed(5)
    rows = A.mx_quantize(torch.randn((K, P), device="cuda"))
    off = torch.arange(T + 1, device="cuda")
    off[T] = P
    _say(f"T={T}")
    v = A.mx_dequantize(rows).double()
    d = (v - v.mean(0)).square().sum(0) / K
    want = torch.cat((d[:T - 1], d[T - 1:].sum()[None]))
    _, var = A.mx_average(rows, off)
    assert bool(((var - want).abs() <= 1e-12 * want).all())
    c = A.mx_product(rows, off)
    # (single products are exact in fp32; the last tensor's are up to 32 sums of 32 each)
    assert torch.equal(c[:T - 1, 0, 1].double(), (v[0] * v[1])[:T - 1]) and torch.equal(c[:, 0, 1], c[:, 1, 0])
    assert torch.equal(c[:T - 1, 1, 1].double(), v[1, :T - 1].square())
    mag = (v[0] * v[1])[T - 1:].abs().sum()
    assert bool((c[T - 1, 0, 1].double() - (v[0] * v[1])[T - 1:].sum()).abs() <= (4 * 32 + 8) * 2.0 ** -24 * mag)


def test_offsets_that_do_not_fit_touch_nothing_else(A):
    """The offsets are read on the device only: boundaries past P, before 0 or out of order leave the
    model right and every other byte as it was."""
    K, P = 4, 10_000
    rng = np.random.default_rng(1)
    codes, byte, v = _message(rng, K, P, ref.E2M1)
    rows = _rows(A, codes, byte, P, ref.E2M1)
    want, _ = A.mx_average(rows, torch.tensor([0, P], device="cuda"))
    for off in ([0, 1 << 40], [-(1 << 40), 5, P], [5000, 100, 9000], [0, 20_000, 30], [7, 7, 7]):
        offd = torch.tensor(off, device="cuda")
        new, var = A.mx_average(rows, offd)
        c = A.mx_product(rows, offd)
        torch.cuda.synchronize()
        assert torch.equal(new, want) and var.shape == (len(off) - 1,) and c.shape == (len(off) - 1, K, K)


@pytest.mark.parametrize("fmt", FORMATS)
def test_replayed_graphs(A, fmt):
    """Two graphs captured from the same buffers, replayed in turn with eager calls between them, give
    the eager bits every time."""
    K, P = 6, 30_011
    rng = np.random.default_rng(11)
    off = torch.tensor([0, 17, 4096, 20_000, P], device="cuda")
    x0 = torch.from_numpy(_numbers(rng, K, P, spread=False)).cuda()
    base0 = torch.zeros(P, device="cuda")
    x, base, res = x0.clone(), base0.clone(), torch.zeros((K, P), device="cuda")
    rows = A.MxRows.empty(K, P, fmt)

    def sync():
        A.mx_quantize(x, base, res, out=rows)
        c = A.mx_product(rows, off)
        _, var = A.mx_average(rows, off, base, x=x, base_out=base)
        return var, c

    def reset(scale):
        x.copy_(x0 * scale)
        base.copy_(base0)
        res.zero_()

    want = {}
    for scale in (1.0, 3.0, 0.1):
        reset(scale)
        var, c = sync()
        want[scale] = [t.clone() for t in (var, c, x, base, res)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sync()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = sync()
        graphs.append((g, out))
    for i, scale in enumerate((1.0, 0.1, 3.0, 1.0, 3.0, 0.1)):
        reset(scale)
        g, (var, c) = graphs[i % 2]
        g.replay()
        torch.cuda.synchronize()
        for got, w in zip((var, c, x, base, res), want[scale]):
            assert torch.equal(got, w)
        reset(0.5)
        sync()
        torch.cuda.synchronize()


@pytest.mark.parametrize("fmt", FORMATS)
def test_another_stream(A, fmt):
    K, P = 8, 200_003
    rng = np.random.default_rng(12)
    x = torch.from_numpy(_numbers(rng, K, P)).cuda()
    off = torch.tensor([0, 100_000, P], device="cuda")
    rows = A.mx_quantize(x, format=fmt)
    want = A.mx_average(rows, off), A.mx_product(rows, off), A.mx_dequantize(rows)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        rows2 = A.mx_quantize(x, format=fmt)
        got = A.mx_average(rows2, off), A.mx_product(rows2, off), A.mx_dequantize(rows2)
    side.synchronize()
    assert torch.equal(got[0][0], want[0][0]) and torch.equal(got[0][1], want[0][1])
    assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])


def test_rows_past_32_bit_offsets(A):
    """Two rows of 1.2e9 elements: bytes and elements past 2^31 and 2^32."""
    K, P = 2, 1_200_000_007
    _say("quantize, average and product of two rows of 1.2e9 elements")
    x = torch.empty((K, P), device="cuda")
    x.normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    rows = A.mx_quantize(x)
    cuts = [0, 1000, P - 2000, P - 33, P]
    off = torch.tensor(cuts, device="cuda")
    new, var = A.mx_average(rows, off)
    c = A.mx_product(rows, off).cpu().numpy()
    y = A.mx_dequantize(rows)
    n = -(-P // 32)
    first = (P - 4096) // 32 * 32
    for a, b in ((0, 4096), (first, P), ((1 << 30) - 64, (1 << 30) + 64)):
        part = x[:, a:b].cpu().numpy()
        _, _, v = ref.quantize(part, ref.E2M1)
        assert _same(y[:, a:b].cpu().numpy(), v)
        assert _same(new[a:b].cpu().numpy(), v.mean(0).astype(np.float32))
        if b == P:
            lo = P - 2000 - a
            want, mag = ref.product(v, v, np.array([lo, P - 33 - a, P - a]))
            assert np.all(np.abs(c[2:] - want) <= _product_tol(np.array([lo, P - 33 - a, P - a]), mag))
            _, wv = ref.average(v[:, lo:], np.array([0, 2000 - 33, 2000]))
            assert np.all(np.abs(var[2:].cpu().numpy() - wv) <= 1e-12 * wv)
    assert rows.codes[1, n * 16 - 16:n * 16].any()
    mean = y.double().mean(0)
    big = slice(1000, P - 2000)
    wv = sum(float(((y[k, big].double() - mean[big]) ** 2).sum()) for k in range(K)) / K
    assert abs(float(var[1]) - wv) <= 1e-10 * wv          # (the reference's own sum of 2.4e9 terms)


@pytest.mark.parametrize("fmt", FORMATS)
def test_error_feedback_keeps_the_sum(A, fmt):
    """Messages and residuals account for everything: after any number of messages the sum of what was
    sent and what is left equals the sum of the differences, to the roundings of the additions."""
    K, P = 3, 10_007
    rng = np.random.default_rng(21)
    res = torch.zeros((K, P), device="cuda")
    sent = torch.zeros((K, P), dtype=torch.float64, device="cuda")
    total = torch.zeros((K, P), dtype=torch.float64, device="cuda")
    most = torch.zeros((K, P), dtype=torch.float64, device="cuda")
    for i in range(5):
        x = torch.from_numpy(_numbers(rng, K, P, spread=False)).cuda()
        most += x.double().abs() + res.double().abs()
        rows = A.mx_quantize(x, None, res, format=fmt)
        sent += A.mx_dequantize(rows).double()
        total += x.double()
    assert bool(((sent + res.double() - total).abs() <= 2.0 ** -24 * most).all())


# ---- the engine's synchronization ------------------------------------------------
def _workload(**kw):
    import workloads as W
    f = dict(name="mx", K=4, sizes=(700, 1, 0, 2500, 33, 5000), seed=9, sigma=0.1, momentum=0.9, weight_decay=5e-4,
             h_lo=1e-2, h_hi=1.0, lr_kind=W.LR_CONST, lr0=0.05, total_steps=60, period_mode=W.PERIOD_ADAPTIVE, p_init=3,
             k_s=15)
    f.update(kw)
    return W.Workload(**f)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("feedback", [True, False])
@pytest.mark.parametrize("pad", [True, False])
def test_engine_sync(A, fmt, feedback, pad):
    """Algorithm 2 by hand with messages in few bits: each sync's model, residual, variances and inner
    products are the reference's of the replicas just before it, and the controller moves as it does
    on the host with the same variances."""
    w = _workload(K=5)
    off, K, P = w.offsets(), w.K, w.P
    base, res = np.zeros(P, np.float32), np.zeros((K, P), np.float32)
    host = A.adpsgd_sched_init(A.hparams_of(w))
    with A.Adpsgd.from_workload(w, pad_rows=pad) as eng:
        t = 0
        while t < w.total_steps:
            p = eng.get_state().p
            eng.local_steps(p)
            for _ in range(p):
                A.adpsgd_sched_step(eng.hp, host)
            t += p
            d = ref.difference(eng.x.cpu().numpy(), base, res if feedback else None)
            m = eng.m.clone()
            _, _, v = ref.quantize(d, fmt)
            new, want = ref.average(v, off, base)
            c, mag = ref.product(v, v, off)
            var, got_c = eng.average_mx(fmt, error_feedback=feedback, products=True)
            assert np.all(np.abs(var - want) <= 1e-12 * want)
            assert np.all(np.abs(got_c - c) <= _product_tol(off, mag))
            got = eng.mx_base.cpu().numpy()
            assert np.all(np.abs(got - new) <= 2.0 ** -24 * (1 + 1e-6) * np.abs(new) + 2.0 ** -149)
            assert _same(eng.x.cpu().numpy(), np.repeat(got[None], K, 0)) and torch.equal(eng.m, m)
            if feedback:
                res = (d - v).astype(np.float32)
                assert _same(eng.mx_residual.cpu().numpy(), res)
            base = got
            assert eng.get_state().cnt == 0
            eng.schedule(var)
            A.adpsgd_sched_on_sync(eng.hp, host, t - 1, float(np.sum(var)))
            st = eng.get_state()
            assert (st.p, st.cnt, st.nC2, st.t) == (host.p, host.cnt, host.nC2, host.t)
        assert host.nC2 > 0 and t >= w.total_steps


def test_engine_sync_on_its_own_stream_and_after_reset(A):
    """On a stream of its own and after reset() the same bits; a change of format in between is allowed."""
    w = _workload(K=3)

    def go(eng, fmts):
        out = []
        for f in fmts:
            eng.local_steps(3)
            out.append(eng.average_mx(f))
        return np.array(out), eng.x.cpu().numpy(), eng.mx_residual.cpu().numpy()

    fmts = [ref.E2M1, ref.E4M3, ref.E2M1]
    with A.Adpsgd.from_workload(w) as eng:
        first = go(eng, fmts)
        eng.reset()
        again = go(eng, fmts)
    with A.Adpsgd.from_workload(w, stream=torch.cuda.Stream()) as eng:
        side = go(eng, fmts)
    for other in (again, side):
        for a, b in zip(first, other):
            assert np.array_equal(a, b)


def test_engine_sync_resumes_bit_exactly(A):
    """A checkpoint of x, m, the controller, mx_base and mx_residual."""
    w = _workload()
    with A.Adpsgd.from_workload(w) as eng:
        for _ in range(3):
            eng.local_steps(4)
            eng.average_mx()
        saved = [t.clone() for t in (eng.x, eng.m, eng.mx_base, eng.mx_residual)], eng.get_state()
        eng.local_steps(4)
        want = eng.average_mx(), eng.x.clone()
    with A.Adpsgd.from_workload(w) as eng:
        eng.average_mx()                       # (of zeros: makes the buffers)
        for t, s in zip((eng.x, eng.m, eng.mx_base, eng.mx_residual), saved[0]):
            t.copy_(s)
        eng.set_state(saved[1])
        eng.local_steps(4)
        assert np.array_equal(eng.average_mx(), want[0]) and torch.equal(eng.x, want[1])


def test_engine_sync_refuses_averaged_momentum(A):
    with A.Adpsgd.from_workload(_workload(avg_momentum=True)) as eng:
        with pytest.raises(ValueError):
            eng.average_mx()


def test_engine_sync_refuses_too_many_products_before_it_sends(A):
    w = _workload(K=257)
    with A.Adpsgd.from_workload(w) as eng:
        eng.local_steps(3)
        x, cnt = eng.x.clone(), eng.get_state().cnt
        with pytest.raises(ValueError):
            eng.average_mx(products=True)
        assert torch.equal(eng.x, x) and eng.get_state().cnt == cnt and eng.mx_residual is None
        eng.average_mx()


def test_rows_keep_what_they_were_made_of(A):
    rows = A.mx_quantize(torch.ones((2, 40), device="cuda"))
    for name in ("codes", "scales", "P", "K", "format"):
        with pytest.raises(AttributeError):
            setattr(rows, name, getattr(rows, name))


def test_tensor_refusals(A):
    """What the Python calls refuse before anything runs."""
    K, P = 3, 100
    x, base = torch.zeros((K, P), device="cuda"), torch.zeros(P, device="cuda")
    rows = A.mx_quantize(x)
    off = torch.tensor([0, P], device="cuda")
    bad = [lambda: A.mx_quantize(x.double()), lambda: A.mx_quantize(x[0]), lambda: A.mx_quantize(x.t()),
           lambda: A.mx_quantize(x[:1].expand(K, P)), lambda: A.mx_quantize(x, base[:-1]),
           lambda: A.mx_quantize(x, base.double()), lambda: A.mx_quantize(x, base.cpu()),
           lambda: A.mx_quantize(x, None, x[:2]), lambda: A.mx_quantize(x, residual_out=base),
           lambda: A.mx_quantize(x, None, torch.zeros((K, P), device="cuda"),
                                 residual_out=torch.zeros((K, P + 1), device="cuda")[:, :P]),
           lambda: A.mx_quantize(x, format=5), lambda: A.mx_quantize(x, format=A.MX_E4M3, out=rows),
           lambda: A.mx_quantize(x[:2], out=rows), lambda: A.mx_quantize(x[:, :64], out=rows),
           lambda: A.mx_dequantize(rows, base[:5]), lambda: A.mx_dequantize(rows, out=x[:2]),
           lambda: A.mx_dequantize(rows, out=x.double()),
           lambda: A.mx_average(rows, off.int()), lambda: A.mx_average(rows, off.cpu()),
           lambda: A.mx_average(rows, off[:1]), lambda: A.mx_average(rows, off[None]),
           lambda: A.mx_average(rows, torch.arange(4, device="cuda")[::2]),
           lambda: A.mx_average(rows, off, base[:5]), lambda: A.mx_average(rows, off, x=x[:2]),
           lambda: A.mx_average(rows, off, base_out=base.double()),
           lambda: A.mx_product(rows, off.float()),
           lambda: A.MxRows(rows.codes, rows.scales, 1_000_000), lambda: A.MxRows(rows.codes.int(), rows.scales, P),
           lambda: A.MxRows(rows.codes, rows.scales[:2], P), lambda: A.MxRows(rows.codes, rows.scales, P, 9),
           lambda: A.MxRows(rows.codes[0], rows.scales[0], P), lambda: A.MxRows(rows.codes, rows.scales, -1),
           lambda: A.MxRows(rows.codes.t(), rows.scales, P)]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            _say(f"refusal {i} did not come")
    lib_bad = [lambda: A.mx_quantize(x, out=A.MxRows(rows.codes[:, 8:72], rows.scales, P)),     # 8 bytes off 16
               lambda: A.mx_quantize(x, residual_out=x), lambda: A.mx_dequantize(rows, x[1], out=x),
               lambda: A.mx_product(rows, off, A.mx_quantize(x, format=A.MX_E4M3)),
               lambda: A.mx_product(A.mx_quantize(torch.zeros((257, 10), device="cuda")), off),
               lambda: A.mx_average(rows, off, x[2], x=x), lambda: A.mx_average(rows, off, x=x, base_out=x[0])]
    for i, f in enumerate(lib_bad):
        with pytest.raises(A.AdpsgdError) as e:
            f()
            _say(f"refusal {i} of the library did not come")
        assert e.value.code == A.EINVAL
