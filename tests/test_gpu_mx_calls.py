"""What the microscaled calls do at the edges of their arguments: rows whose numbers pass fp32,
what is refused before memory is taken for it, tensors that take part in autograd, sums of products of many sizes."""
import numpy as np
import pytest
import torch

import mx_reference as ref
from test_gpu_mx import _rows, _same

pytestmark = pytest.mark.gpu

FORMATS = [ref.E2M1, ref.E4M3]


@pytest.fixture(scope="module")
def A():
    assert torch.cuda.is_available()
    import paper_2007_06134_amd as A
    return A


def _far_rows(rng, K, P, fmt):
    """Codes and scale bytes as a sender of another make may have them: all codes but NaN, scales up to
    2^127, so that many numbers pass fp32; ordinary and NaN blocks among them."""
    n = -(-P // 32)
    codes = rng.integers(0, 256, (K, n * (16 if fmt == ref.E2M1 else 32)), dtype=np.uint8)
    if fmt == ref.E4M3:
        codes[codes % 128 == 127] = 0x7E
    byte = rng.integers(240, 255, (K, n)).astype(np.uint8)
    byte[:, rng.random(n) < 0.3] = 127
    byte[K - 1, n // 2] = 255
    return codes, byte


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("K,P", [(2, 33), (4, 3001), (9, 70_001), (17, 2000), (2, 4_300_001)])
def test_average_of_numbers_past_fp32(A, fmt, K, P):
    """Their sums are 64-bit ones, so opposite numbers of 2^128 and more cancel; what does not fit is an
    infinity in the model only."""
    rng = np.random.default_rng([fmt, K, P, 5])
    codes, byte = _far_rows(rng, K, P, fmt)
    if K % 2 == 0:       # half of the workers send the other half's negatives, but for one element
        h = K // 2
        codes[h:] = codes[:h] ^ (0x88 if fmt == ref.E2M1 else 0x80)
        byte[h:] = byte[:h]
        byte[K - 1, 0] = 127
    v = ref.values(codes, byte, P, fmt)
    off = np.array([0, 3, 3, 32, P])
    base = rng.standard_normal(P).astype(np.float32)
    rows, offd = _rows(A, codes, byte, P, fmt), torch.from_numpy(off).cuda()
    for b in (None, base):
        new, want = ref.average(v, off, b)
        x = torch.empty((K, P), device="cuda")
        got, var = A.mx_average(rows, offd, None if b is None else torch.from_numpy(b).cuda(), x=x)
        got, var = got.cpu().numpy().astype(np.float64), var.cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(new)) and np.array_equal(np.isnan(var), np.isnan(want))
        ok = ~np.isnan(new)
        most = np.float64(np.finfo(np.float32).max)
        fits = ok & (np.abs(new) <= most)
        past = ok & (np.abs(new) >= 2.0 ** 128 * (1 - 2.0 ** -25))
        # (a mean of K numbers that are not powers of two apart is rounded in 64 bits first)
        assert np.all(np.abs(got - new)[fits] <= 2.0 ** -24 * (1 + 1e-6) * np.abs(new)[fits] + 2.0 ** -149)
        assert np.all(np.isinf(got[past])) and np.all(np.signbit(got[past]) == np.signbit(new[past]))
        ok = ~np.isnan(want)
        assert ok.any() and np.all(np.abs(var - want)[ok] <= 1e-12 * want[ok])
        assert _same(x.cpu().numpy(), np.repeat(got[None].astype(np.float32), K, 0))
    if K % 2 == 0:
        assert np.all(new[~np.isnan(new)][40:] == base[~np.isnan(new)][40:])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("K", [1, 3, 7])
def test_read_back_of_numbers_past_fp32(A, fmt, K):
    """base + number, rounded once: finite where the sum is."""
    P = 5000
    rng = np.random.default_rng([fmt, K, 6])
    codes, byte = _far_rows(rng, K, P, fmt)
    v = ref.values(codes, byte, P, fmt)
    base = (rng.uniform(-1, 1, P) * 2.0 ** 128 * (1 - 2.0 ** -24)).astype(np.float32)
    rows = _rows(A, codes, byte, P, fmt)
    with np.errstate(over="ignore"):
        assert _same(A.mx_dequantize(rows).cpu().numpy(), v.astype(np.float32))
        want = base.astype(np.float64) + v
        rescued = (np.abs(v) >= 2.0 ** 128) & (np.abs(want) < 2.0 ** 127)
        assert rescued.sum() > 10
        assert _same(A.mx_dequantize(rows, torch.from_numpy(base).cuda()).cpu().numpy(), want.astype(np.float32))


def test_four_bit_products_of_numbers_past_fp32(A):
    """The matrix instruction applies both scales to the product: 6 * 2^127 against numbers near 2^-127."""
    P = 64
    rng = np.random.default_rng(3)
    codes = rng.integers(0, 256, (2, 4, P // 2), dtype=np.uint8)
    byte = np.stack([np.full((4, 2), 254, np.uint8), np.array([[0, 0], [1, 1], [2, 0], [120, 121]], np.uint8)])
    v, w = (ref.values(codes[i], byte[i], P, ref.E2M1) for i in range(2))
    got = A.mx_product(_rows(A, codes[0], byte[0], P, ref.E2M1), torch.tensor([0, P], device="cuda"),
                       _rows(A, codes[1], byte[1], P, ref.E2M1)).cpu().numpy()[0]
    assert np.array_equal(got.astype(np.float64), v @ w.T)       # (quarters of integers up to 144, under few scales)


def test_eight_bit_products_of_numbers_past_fp32(A):
    """The operands are bf16 numbers: those of 2^128 and more count as infinite, so their products do."""
    P = 32
    codes = np.full((2, 1, P), 0x38, np.uint8)        # 1
    codes[0, 0, 3] = 0x7E                             # 448
    byte = np.array([[[246]], [[127]]], np.uint8)     # 448 * 2^119 < 2^128
    offs = torch.tensor([0, P], device="cuda")
    other = _rows(A, codes[1], byte[1], P, ref.E4M3)
    got = A.mx_product(_rows(A, codes[0], byte[0], P, ref.E4M3), offs, other).item()
    assert got == 479 * 2.0 ** 119
    got = A.mx_product(_rows(A, codes[0], byte[0] + 8, P, ref.E4M3), offs, other).item()
    assert got == np.inf


def _allocations():
    return torch.cuda.memory_stats()["allocation.all.allocated"]


def test_what_the_library_refuses_takes_no_memory(A):
    """Thousands of workers' products, or more rows than a call takes: the refusal, not a failed
    allocation of what the call would have written."""
    off = torch.tensor([0, 10], device="cuda")
    many = A.MxRows(torch.zeros((3000, 16), dtype=torch.uint8, device="cuda"),
                    torch.zeros((3000, 16), dtype=torch.uint8, device="cuda"), 10)
    n = _allocations()
    with pytest.raises(A.AdpsgdError, match="256") as e:
        A.mx_product(many, off)
    assert e.value.code == A.EINVAL and _allocations() == n
    one = A.mx_quantize(torch.zeros((4, 10), device="cuda"))
    two = A.mx_quantize(torch.zeros((4, 10), device="cuda"), format=A.MX_E4M3)
    n = _allocations()
    with pytest.raises(A.AdpsgdError, match="same format"):
        A.mx_product(one, off, two)
    assert _allocations() == n
    x, b = torch.zeros((65537, 1), device="cuda"), torch.zeros((65537, 16), dtype=torch.uint8, device="cuda")
    n = _allocations()
    for call in (lambda: A.mx_quantize(x), lambda: A.MxRows(b, b, 1)):
        with pytest.raises(ValueError, match="65536"):
            call()
    assert _allocations() == n


def _calls(A, K=3, P=100):
    """(name, call with that tensor, the tensor) of every float tensor that a call takes."""
    z = lambda *s: torch.zeros(s, device="cuda")      # noqa: E731
    off = torch.tensor([0, P], device="cuda")
    rows = A.mx_quantize(z(K, P))
    return [("x", lambda t: A.mx_quantize(t), z(K, P)), ("base", lambda t: A.mx_quantize(z(K, P), t), z(P)),
            ("residual", lambda t: A.mx_quantize(z(K, P), None, t), z(K, P)),
            ("residual_out", lambda t: A.mx_quantize(z(K, P), residual_out=t), z(K, P)),
            ("base", lambda t: A.mx_dequantize(rows, t), z(P)), ("out", lambda t: A.mx_dequantize(rows, out=t), z(K, P)),
            ("base", lambda t: A.mx_average(rows, off, t), z(P)), ("x", lambda t: A.mx_average(rows, off, x=t), z(K, P)),
            ("base_out", lambda t: A.mx_average(rows, off, base_out=t), z(P))]


def test_tensors_that_record_gradients_are_refused(A):
    """No gradient flows through the calls: silently cutting the graph is an error, under no_grad it is asked for."""
    for name, call, t in _calls(A):
        t.requires_grad_()
        with pytest.raises(ValueError, match=name + ".*no_grad"):
            call(t)
        with torch.no_grad():
            call(t)


def test_writes_under_no_grad_are_seen_by_autograd(A):
    """A parameter that an earlier graph saved and a call then writes: its backward raises, as after torch's own
    writes, in place of taking the new values."""
    for name, call, t in _calls(A):
        t.requires_grad_()
        y = (t * t).sum()
        with torch.no_grad():
            call(t)
        # (residual is written where there is no residual_out)
        if name in ("residual", "residual_out", "out", "base_out") or (name == "x" and t._version):
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                y.backward()
        else:
            y.backward()
    t = torch.zeros((3, 100), device="cuda", requires_grad=True)
    rows, off = A.mx_quantize(torch.ones((3, 100), device="cuda")), torch.tensor([0, 100], device="cuda")
    before = t._version
    with torch.no_grad():
        A.mx_average(rows, off, x=t)
    assert t._version > before


# of a result whose products are all positive: a level of 512 elements is 4 matrix instructions of at most four
# roundings, then at most 32 of those sums, the partial sum's rounding and the result's
_LEVELS = (4 * 4 + 32 + 2) * 2.0 ** -24


@pytest.mark.parametrize("K", [1, 2, 4, 8, 16, 32, 48, 64, 70])
def test_four_bit_products_of_blocks_of_many_sizes(A, K):
    """Blocks whose sizes differ by a decade or so: sums of few products are no longer exact."""
    P = 600_000
    g = torch.Generator(device="cuda").manual_seed(K)
    size = torch.exp(2.3 * torch.randn((K, P // 32), device="cuda", generator=g)).repeat_interleave(32, 1)
    x = size * (torch.rand((K, P), device="cuda", generator=g) + 0.1)
    rows = A.mx_quantize(x)
    v = A.mx_dequantize(rows).double()
    got = A.mx_product(rows, torch.tensor([0, P], device="cuda"))[0].double()
    want = v @ v.t().contiguous()
    off_by = ((got - want).abs() / want).max().item()
    print(f"K={K}: {off_by:.2e} of the result")
    assert off_by <= _LEVELS


@pytest.mark.parametrize("K,P", [(8, 168_000_000), (16, 84_000_000), (32, 34_000_000), (64, 17_000_000), (70, 8_400_000)])
def test_four_bit_products_keep_small_terms_beside_a_large_one(A, K, P):
    """Every 16384 elements a 1, the rest 2^-16: 128 of their products are less than half a step of a sum that
    holds the 1, 512 of them are a step of it.  One sum of 16384 products would lose 16352 * 2^-32, 3.8e-6."""
    P -= P % 16384
    codes = torch.full((K, P // 2), 0x22, dtype=torch.uint8, device="cuda")       # ones
    scales = torch.full((K, P // 32), 127 - 16, dtype=torch.uint8, device="cuda")
    scales[:, ::512] = 127
    codes.view(K, -1, 16)[:, ::512] = 0
    codes.view(K, -1, 16)[:, ::512, 0] = 0x02
    got = A.mx_product(A.MxRows(codes, scales, P), torch.tensor([0, P], device="cuda"))[0].double().cpu()
    want = (P // 16384) * (1 + 16352 * 2.0 ** -32)
    print(f"K={K}: {((got - want).abs().max() / want).item():.2e} of the result")
    assert bool(((got - want).abs() <= _LEVELS * want).all())
