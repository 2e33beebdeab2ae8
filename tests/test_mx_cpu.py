"""The microscaled messages without a GPU: refusals of the C calls (nothing is launched), strides,
workspaces, and the test reference itself."""
import ctypes as C

import numpy as np
import pytest
import torch

import mx_reference as ref


@pytest.fixture(scope="module")
def A():
    import paper_2007_06134_amd as A
    return A


@pytest.fixture(scope="module")
def lib(A):
    return A._native.lib


BASE = 1 << 20        # host numbers standing in for device addresses: validation reads no memory


def _rows(A, **kw):
    f = dict(codes=BASE, scales=BASE, code_stride=256, scale_stride=256, P=100, K=4, format=0)
    f.update(kw)
    return A.adpsgd_mx_rows(**f)


BAD_ROWS = [dict(format=2), dict(format=-1), dict(K=0), dict(K=65537), dict(K=-3), dict(P=-1), dict(P=1 << 40),
            dict(P=1 << 34, K=1 << 16, code_stride=1 << 34, scale_stride=1 << 30),
            dict(code_stride=48), dict(code_stride=63), dict(code_stride=72), dict(code_stride=64, format=1),
            dict(code_stride=-256), dict(scale_stride=0), dict(scale_stride=3), dict(scale_stride=20),
            dict(codes=0), dict(scales=0), dict(codes=BASE + 8), dict(scales=BASE + 4)]


@pytest.mark.parametrize("bad", BAD_ROWS)
def test_rows_are_checked_by_every_call(A, lib, bad):
    r, good = _rows(A, **bad), _rows(A)
    ref_ = C.byref
    calls = [lambda: lib.adpsgd_mx_quantize(ref_(r), BASE, 0, None, None, None, 0, None),
             lambda: lib.adpsgd_mx_dequantize(ref_(r), None, BASE, 0, None),
             lambda: lib.adpsgd_mx_average(ref_(r), 1, BASE, None, BASE, None, 0, BASE, BASE, 1 << 30, None),
             lambda: lib.adpsgd_mx_product(ref_(r), None, 1, BASE, BASE, BASE, 1 << 30, None),
             lambda: lib.adpsgd_mx_product(ref_(good), ref_(r), 1, BASE, BASE, BASE, 1 << 30, None)]
    for call in calls:
        assert call() == A.EINVAL and A.adpsgd_last_error()


@pytest.mark.parametrize("K", [1, 4])
def test_strides_whose_addresses_would_not_fit_are_refused(A, lib, K):
    far, huge = 1 << 60, (1 << 44) + 16
    for ld in (far, huge, (1 << 63) - 1):
        r = C.byref(_rows(A, K=K))
        calls = [lambda: lib.adpsgd_mx_quantize(r, BASE, ld, None, None, None, 0, None),
                 lambda: lib.adpsgd_mx_quantize(r, BASE, 0, None, BASE, None, ld, None),
                 lambda: lib.adpsgd_mx_dequantize(r, None, BASE, ld, None),
                 lambda: lib.adpsgd_mx_average(r, 1, BASE, None, None, BASE, ld, BASE, BASE, 1 << 20, None)]
        for name in ("code_stride", "scale_stride"):
            if ld % 16 == 0:
                bad = C.byref(_rows(A, K=K, **{name: ld}))
                calls.append(lambda bad=bad: lib.adpsgd_mx_product(bad, None, 1, BASE, BASE, BASE, 1 << 30, None))
        for call in calls:
            assert call() == A.EINVAL and "2^44" in A.adpsgd_last_error()


@pytest.mark.parametrize("P", [(1 << 34) + 1, (1 << 63) - 4, (1 << 63) - 1])
def test_lengths_past_the_limit_are_refused(A, lib, P):
    """Also those whose bytes or blocks no 64-bit count holds."""
    r = C.byref(_rows(A, P=P, K=1, code_stride=1 << 43, scale_stride=1 << 43))
    for call in (lambda: lib.adpsgd_mx_quantize(r, BASE, 0, None, None, None, 0, None),
                 lambda: lib.adpsgd_mx_dequantize(r, None, BASE, 0, None),
                 lambda: lib.adpsgd_mx_average(r, 1, BASE, None, BASE, None, 0, BASE, BASE, 1 << 60, None),
                 lambda: lib.adpsgd_mx_product(r, None, 1, BASE, BASE, BASE, 1 << 60, None)):
        assert call() == A.EINVAL and "P must" in A.adpsgd_last_error()
    assert lib.adpsgd_mx_average_workspace(1, P, 1) == 0 and lib.adpsgd_mx_product_workspace(1, P, 1) == 0
    for fmt in (A.MX_E2M1, A.MX_E4M3):
        assert lib.adpsgd_mx_code_stride(fmt, P) == 0
        with pytest.raises(ValueError):
            A.MxRows.empty(1, P, fmt, device="cpu")
    assert lib.adpsgd_mx_scale_stride(P) == 0


def test_null_rows(A, lib):
    assert lib.adpsgd_mx_quantize(None, BASE, 0, None, None, None, 0, None) == A.EINVAL
    assert lib.adpsgd_mx_dequantize(None, None, BASE, 0, None) == A.EINVAL
    assert lib.adpsgd_mx_average(None, 1, BASE, None, BASE, None, 0, BASE, BASE, 1 << 30, None) == A.EINVAL
    assert lib.adpsgd_mx_product(None, None, 1, BASE, BASE, BASE, 1 << 30, None) == A.EINVAL


@pytest.mark.parametrize("args,word", [
    ((None, 0, None, None, None, 0), "x must"), ((BASE + 2, 0, None, None, None, 0), "x must"),
    ((BASE, 99, None, None, None, 0), "x_stride"), ((BASE, -1, None, None, None, 0), "x_stride"),
    ((BASE, 0, BASE + 1, None, None, 0), "base"), ((BASE, 0, None, BASE + 3, None, 0), "residual_in"),
    ((BASE, 0, None, None, BASE + 1, 0), "residual_out"), ((BASE, 0, None, BASE, BASE, 99), "residual_stride"),
    ((BASE, 0, None, BASE, BASE, -5), "residual_stride"),
])
def test_quantize_refuses(A, lib, args, word):
    assert lib.adpsgd_mx_quantize(C.byref(_rows(A)), *args, None) == A.EINVAL
    assert word in A.adpsgd_last_error()


def test_residuals_that_lie_across_each_other_are_refused(A, lib):
    """residual_out is residual_in or apart from it: rows that begin elsewhere in it would be read
    after they were written.  The same for the inputs x and base."""
    r = C.byref(_rows(A))                                     # 4 rows of 100 elements
    for other in (BASE + 4, BASE + 400, BASE - 400, BASE + 1596):
        assert lib.adpsgd_mx_quantize(r, 1 << 30, 0, None, BASE, other, 0, None) == A.EINVAL
        assert "overlap" in A.adpsgd_last_error()
    for x, base in ((BASE + 400, None), (1 << 30, BASE + 396)):
        assert lib.adpsgd_mx_quantize(r, x, 0, base, None, BASE, 0, None) == A.EINVAL
        assert "overlap" in A.adpsgd_last_error()


@pytest.mark.parametrize("args,word", [((None, None, 0), "y must"), ((None, BASE + 2, 0), "y must"),
                                       ((BASE + 2, BASE, 0), "base"), ((None, BASE, 99), "y_stride")])
def test_dequantize_refuses(A, lib, args, word):
    assert lib.adpsgd_mx_dequantize(C.byref(_rows(A)), *args, None) == A.EINVAL
    assert word in A.adpsgd_last_error()


def test_a_base_inside_the_rows_written_is_refused(A, lib):
    r = C.byref(_rows(A))
    assert lib.adpsgd_mx_dequantize(r, BASE + 400, BASE, 0, None) == A.EINVAL
    assert "overlap" in A.adpsgd_last_error()
    big = dict(workspace=1 << 40, n=1 << 30)
    for base, base_out, x in ((BASE, BASE + 4, None), (BASE, None, BASE + 4), (None, BASE, BASE + 1200)):
        rc = lib.adpsgd_mx_average(r, 1, 1 << 35, base, base_out, x, 0, 1 << 36, big["workspace"], big["n"], None)
        assert rc == A.EINVAL and "overlap" in A.adpsgd_last_error()


@pytest.mark.parametrize("T,off,base,base_out,x,x_ld,var,ws,n,word", [
    (0, BASE, None, None, None, 0, BASE, BASE, 1 << 20, "T must"),
    ((1 << 24) + 1, BASE, None, None, None, 0, BASE, BASE, 1 << 40, "T must"),
    (1, None, None, None, None, 0, BASE, BASE, 1 << 20, "tensor_offsets"),
    (1, BASE + 4, None, None, None, 0, BASE, BASE, 1 << 20, "tensor_offsets"),
    (1, BASE, BASE + 2, None, None, 0, BASE, BASE, 1 << 20, "base"),
    (1, BASE, None, BASE + 2, None, 0, BASE, BASE, 1 << 20, "base_out"),
    (1, BASE, None, None, BASE + 2, 0, BASE, BASE, 1 << 20, "x must"),
    (1, BASE, None, None, BASE, 99, BASE, BASE, 1 << 20, "x_stride"),
    (1, BASE, None, None, None, 0, None, BASE, 1 << 20, "var"),
    (1, BASE, None, None, None, 0, BASE + 4, BASE, 1 << 20, "var"),
    (1, BASE, None, None, None, 0, BASE, None, 1 << 20, "workspace"),
    (1, BASE, None, None, None, 0, BASE, BASE + 128, 1 << 20, "workspace"),
    (1, BASE, None, None, None, 0, BASE, BASE, 1, "workspace"),
])
def test_average_refuses(A, lib, T, off, base, base_out, x, x_ld, var, ws, n, word):
    assert lib.adpsgd_mx_average(C.byref(_rows(A)), T, off, base, base_out, x, x_ld, var, ws, n, None) == A.EINVAL
    assert word in A.adpsgd_last_error()


def test_product_refuses(A, lib):
    def call(a, b, T=1, off=BASE, out=BASE, ws=BASE, n=1 << 30):
        return lib.adpsgd_mx_product(C.byref(a), C.byref(b) if b is not None else None, T, off, out, ws, n, None)
    a = _rows(A)
    for b in (_rows(A, codes=2 * BASE, format=1), _rows(A, codes=2 * BASE, K=3), _rows(A, codes=2 * BASE, P=99)):
        assert call(a, b) == A.EINVAL and "same format" in A.adpsgd_last_error()
    assert call(a, _rows(A, code_stride=512)) == A.EINVAL          # the same memory, other rows
    assert call(_rows(A, K=257), None) == A.EINVAL and "256" in A.adpsgd_last_error()
    assert call(a, None, T=0) == A.EINVAL
    assert call(a, None, off=None) == A.EINVAL
    assert call(a, None, out=None) == A.EINVAL and call(a, None, out=BASE + 2) == A.EINVAL
    assert call(a, None, ws=None) == A.EINVAL and call(a, None, ws=BASE + 64) == A.EINVAL
    assert call(a, None, n=lib.adpsgd_mx_product_workspace(4, 100, 1) - 1) == A.EINVAL


def test_strides_and_workspaces(A, lib):
    for fmt, per in ((A.MX_E2M1, 16), (A.MX_E4M3, 32)):
        for P in (1, 31, 32, 33, 511, 512, 100_000, 138_000_000):
            n = -(-P // 32)
            for s, need in ((lib.adpsgd_mx_code_stride(fmt, P), n * per), (lib.adpsgd_mx_scale_stride(P), n)):
                assert s >= need and s % 256 == 0 and (s // 256) % 2 == 1 and s - need < 512
    assert lib.adpsgd_mx_code_stride(2, 100) == 0 and lib.adpsgd_mx_code_stride(0, 0) == 0
    assert lib.adpsgd_mx_scale_stride(-1) == 0
    for f, K in ((lib.adpsgd_mx_average_workspace, 65536), (lib.adpsgd_mx_product_workspace, 256)):
        assert f(K, 1000, 1) > 0 and f(1, 0, 1) > 0
        assert f(0, 1000, 1) == 0 and f(K + 1, 1000, 1) == 0 and f(4, -1, 1) == 0 and f(4, 1 << 40, 1) == 0
        assert f(4, 1000, 0) == 0 and f(4, 1000, (1 << 24) + 1) == 0


def test_tensors_on_the_cpu_are_refused(A):
    cpu = torch.zeros((2, 64), dtype=torch.uint8)
    with pytest.raises(ValueError):
        A.MxRows(cpu, cpu, 32)
    with pytest.raises(ValueError):
        A.mx_quantize(torch.zeros(2, 64))
    with pytest.raises(ValueError):
        A.MxRows.empty(0, 5)
    with pytest.raises(ValueError):
        A.MxRows.empty(2, 5, format=7)


# ---- the reference: grids by hand, rounding against brute force ----------------
def test_reference_grids():
    assert ref.grid(ref.E2M1).tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    want = torch.arange(128, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.grid(ref.E4M3), want, equal_nan=True)


@pytest.mark.parametrize("fmt", [ref.E2M1, ref.E4M3])
def test_reference_rounds_to_the_nearest(fmt):
    rng = np.random.default_rng(0)
    d = (rng.standard_normal((3, 200)) * 10.0 ** rng.uniform(-5, 5, (3, 200))).astype(np.float32)
    codes, byte, v = ref.quantize(d, fmt)
    g = ref.grid(fmt)[:8 if fmt == ref.E2M1 else 127]
    full = np.concatenate([g, -g])
    for k in range(3):
        for i in range(200):
            b = d[k, i // 32 * 32:i // 32 * 32 + 32].astype(np.float64)
            s = 2.0 ** (int(byte[k, i // 32]) - 127)
            assert np.abs(b).max() <= g[-1] * s and np.abs(b).max() > g[-1] * s / 2
            assert abs(v[k, i] - d[k, i]) == np.abs(full * s - np.float64(d[k, i])).min()
    packed = ref.pack(codes, fmt)
    assert np.array_equal(ref.values(packed, byte, 200, fmt), v)


def test_reference_ties_go_to_the_even_code():
    d = np.zeros((1, 32), np.float32)
    d[0, :8] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5]
    assert ref.quantize(d, ref.E2M1)[2][0, :8].tolist() == [6, 0, 1, 1, 2, 2, 4, 4]
