"""Microscaled matrices, what needs no GPU: the oracle's format, the pitches, and every refusal
(all of them are found on the host before anything is launched)."""
import contextlib
import ctypes
import math
import types

import numpy as np
import pytest

from oracle import mx as om


def test_format_tables():
    v4, v8 = om.format_values(4), om.format_values(8)
    assert list(v4[:8]) == [0, 0.5, 1, 1.5, 2, 3, 4, 6] and list(v4[8:]) == [-v for v in v4[:8]]
    assert v8[1] == 2.0 ** -9 and v8[8] == 2.0 ** -6 and v8[0x7E] == 448 and math.isnan(v8[0x7F]) and math.isnan(v8[0xFF])
    assert np.all(np.diff(v8[:0x7F]) > 0)
    torch = pytest.importorskip("torch")
    t = torch.arange(256).to(torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(t, v8, equal_nan=True)


def test_oracle_rounds_to_even_and_cuts_down():
    # a maximum of 4 makes the scale 1; of 7.9 too
    row = np.array([[4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, -0.25, -5.0, 0.26, 0.2500001, 2.49]])
    c, s = om.quantize(row, 4)
    assert s[0, 0] == 127
    got = om.values(c, s, row.shape[1], 4)[0]
    assert list(got) == [4, 0, 1, 1, 2, 2, 4, 0, -4, 0.5, 0.5, 2]
    c, s = om.quantize(np.array([[7.9, -7.9, 5.0, 5.1]]), 4)
    assert s[0, 0] == 127 and list(om.values(c, s, 4, 4)[0]) == [6, -6, 4, 6]
    c, s = om.quantize(np.array([[511.0, 17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10]]), 8)
    assert s[0, 0] == 127 and list(om.values(c, s, 5, 8)[0]) == [448, 16, 20, 0, 2.0 ** -8]
    c, s = om.quantize(np.array([[1.0, np.inf] + [0.0] * 30 + [2.0]]), 4)
    assert list(s[0]) == [255, 126] and np.all(np.isnan(om.values(c, s, 33, 4)[0, :32]))
    c, s = om.quantize(np.array([[0.0, 1e-45]]), 8)
    assert s[0, 0] == 10


@pytest.mark.parametrize("r,pitch4,scale", [(0, 0, 0), (1, 16, 4), (32, 16, 4), (33, 32, 4), (128, 64, 4), (129, 80, 8), (5750, 2880, 180)])
def test_sizes(lib, r, pitch4, scale):
    assert lib.coded_mx_sizes(lib.CODED_MX4, r) == (pitch4, scale)
    assert lib.coded_mx_sizes(lib.CODED_MX8, r) == (2 * pitch4, scale)


def test_sizes_refused(lib):
    for fmt, r, status in [(lib.CODED_BF16, 5, lib.CODED_ERR_ARG), (99, 5, lib.CODED_ERR_ARG), (lib.CODED_MX4, -1, lib.CODED_ERR_SHAPE)]:
        with pytest.raises(lib.CodedError) as e:
            lib.coded_mx_sizes(fmt, r)
        assert e.value.status == status


# A 6 x 40 matrix in 4 bits (pitches 32 and 4) with two right-hand sides: addresses that the checks
# look at and nothing reads.
GOOD = dict(fmt=3, codes=0x1000, ldc=32, scales=0x2000, lds=4, q=6, r=40, x_dt=0, X=0x3000, ldx=2, xs=None, ldxs=0, s=2,
            order=0, alpha=1.0, beta=0.0, C=None, ldcc=0, Y=0x4000, y_dt=0, ldy=2, ws=None, wsb=0)

BAD = [
    (dict(fmt=0), "ARG"), (dict(fmt=2), "ARG"), (dict(fmt=77), "ARG"),
    (dict(codes=None), "ARG"), (dict(scales=None), "ARG"), (dict(codes=0x1008), "ARG"), (dict(scales=0x2002), "ARG"),
    (dict(ldc=16), "SHAPE"), (dict(ldc=40), "SHAPE"), (dict(ldc=-32), "SHAPE"), (dict(lds=0), "SHAPE"), (dict(lds=6), "SHAPE"),
    (dict(q=-1), "SHAPE"), (dict(r=-1), "SHAPE"), (dict(s=-1), "SHAPE"), (dict(q=2 ** 41), "SHAPE"), (dict(s=2 ** 41), "SHAPE"),
    (dict(x_dt=2), "ARG"), (dict(x_dt=9), "ARG"), (dict(X=None), "ARG"), (dict(X=0x3002), "ARG"), (dict(ldx=1), "SHAPE"),
    (dict(order=4), "ARG"), (dict(order=-1), "ARG"), (dict(order=1, ldx=39), "SHAPE"), (dict(order=2, ldy=5), "SHAPE"),
    (dict(Y=None), "ARG"), (dict(Y=0x4001), "ARG"), (dict(y_dt=2), "ARG"), (dict(ldy=1), "SHAPE"),
    (dict(alpha=math.inf), "ARG"), (dict(alpha=math.nan), "ARG"), (dict(beta=math.nan), "ARG"),
    (dict(beta=1.0), "ARG"), (dict(beta=1.0, C=0x5000, ldcc=1), "SHAPE"), (dict(beta=1.0, C=0x5000, ldcc=-2), "SHAPE"),
    (dict(beta=1.0, C=0x5002, ldcc=2), "ARG"), (dict(beta=1.0, C=0x4000, ldcc=0), "ARG"),
]
BAD_MM = [
    (dict(x_dt=3, ldx=32, xs=0x6000, ldxs=4), "UNSUPPORTED"), (dict(x_dt=3, ldx=16, xs=0x6000, ldxs=4, order=1), "SHAPE"),
    (dict(x_dt=4, ldx=32, xs=0x6000, ldxs=4, order=1), "SHAPE"), (dict(x_dt=3, ldx=32, order=1), "SHAPE"),
    (dict(x_dt=3, ldx=32, ldxs=4, order=1), "ARG"), (dict(x_dt=3, X=0x3004, ldx=32, xs=0x6000, ldxs=4, order=1), "ARG"),
]


def _call(lib, transposed, **change):
    a = {**GOOD, **change}
    if transposed and "ldy" not in change and a["order"] & 2:
        a["ldy"] = 40
    h = lib.lib()
    common = (a["fmt"], a["codes"], a["ldc"], a["scales"], a["lds"], a["q"], a["r"], a["x_dt"], a["X"], a["ldx"])
    tail = (a["s"], a["order"], a["alpha"], a["beta"], a["C"], a["ldcc"], a["Y"], a["y_dt"], a["ldy"], a["ws"], a["wsb"], None)
    if transposed:
        return h.coded_mx_mm_t(*common, *tail)
    return h.coded_mx_mm(*common, a["xs"], a["ldxs"], *tail)


@pytest.mark.parametrize("change,status", BAD + BAD_MM)
def test_product_refused(lib, change, status):
    assert _call(lib, False, **change) == getattr(lib, "CODED_ERR_" + status)
    assert lib.last_error()


@pytest.mark.parametrize("change,status", [b for b in BAD if "ldx" not in b[0] and "ldy" not in b[0]] + [
    (dict(ldx=1), "SHAPE"), (dict(order=1, ldx=5), "SHAPE"), (dict(order=2, ldy=39), "SHAPE"), (dict(x_dt=3), "ARG"), (dict(x_dt=4), "ARG")])
def test_transposed_product_refused(lib, change, status):
    assert _call(lib, True, **change) == getattr(lib, "CODED_ERR_" + status)
    assert lib.last_error()


def test_nothing_to_write_is_fine_without_a_gpu(lib):
    for transposed in (False, True):
        assert _call(lib, transposed, s=0) == lib.CODED_OK
        assert _call(lib, transposed, **{"r" if transposed else "q": 0}) == lib.CODED_OK


def test_storing_refused(lib):
    h = lib.lib()
    good = dict(dt=0, A=0x1000, q=3, r=40, lda=40, fmt=3, codes=0x2000, ldc=32, scales=0x3000, lds=4)
    for change, status in [(dict(dt=2), "ARG"), (dict(dt=3), "ARG"), (dict(A=None), "ARG"), (dict(A=0x1002), "ARG"), (dict(lda=39), "SHAPE"),
                           (dict(fmt=1), "ARG"), (dict(codes=None), "ARG"), (dict(codes=0x2004), "ARG"), (dict(ldc=31), "SHAPE"),
                           (dict(ldc=16), "SHAPE"), (dict(scales=None), "ARG"), (dict(lds=2), "SHAPE"), (dict(q=-1), "SHAPE"),
                           (dict(r=-5), "SHAPE"), (dict(fmt=4), "SHAPE")]:
        a = {**good, **change}
        st = h.coded_mx_quantize(a["dt"], a["A"], a["q"], a["r"], a["lda"], a["fmt"], a["codes"], a["ldc"], a["scales"], a["lds"], None)
        assert st == getattr(lib, "CODED_ERR_" + status), change
        st = h.coded_mx_dequantize(a["fmt"], a["codes"], a["ldc"], a["scales"], a["lds"], a["q"], a["r"], a["dt"], a["A"], a["lda"], None)
        assert st == getattr(lib, "CODED_ERR_" + status), change
    for change in (dict(q=0), dict(r=0)):
        a = {**good, **change}
        assert h.coded_mx_quantize(a["dt"], a["A"], a["q"], a["r"], a["lda"], a["fmt"], a["codes"], a["ldc"], a["scales"], a["lds"], None) == lib.CODED_OK


def test_workspace_refused(lib):
    b = ctypes.c_int64()
    at = ctypes.addressof(b)
    h = lib.lib()
    assert h.coded_mx_workspace(0, 3, 64, 64, 0, 1, 0, at) == lib.CODED_OK and b.value >= 0
    assert h.coded_mx_workspace(0, 3, 64, 64, 4, 1, 1, at) == lib.CODED_OK
    for args, status in [((0, 0, 64, 64, 0, 1, 0, at), "ARG"), ((0, 3, 64, 64, 2, 1, 0, at), "ARG"), ((1, 3, 64, 64, 3, 1, 1, at), "ARG"),
                         ((0, 3, -1, 64, 0, 1, 0, at), "SHAPE"), ((0, 3, 64, 64, 0, 1, 8, at), "ARG"), ((0, 3, 64, 64, 0, 1, 0, None), "ARG")]:
        assert h.coded_mx_workspace(*args) == getattr(lib, "CODED_ERR_" + status), args


def test_binding_refuses_wrong_tensors(lib):
    torch = pytest.importorskip("torch")
    M = lib.alloc_mx(6, 40, lib.CODED_MX4, device="cpu")
    assert M.shape == (6, 40) and M.rows(2, 5).shape == (3, 40)
    with pytest.raises(ValueError):
        lib.MXMatrix(M.codes, M.scales, 41 + 32, lib.CODED_MX4)
    with pytest.raises(ValueError):
        lib.MXMatrix(M.codes, M.scales, 40, lib.CODED_MX8)
    with pytest.raises(ValueError):
        lib.MXMatrix(M.codes, M.scales[:5], 40, lib.CODED_MX4)
    with pytest.raises(ValueError):
        lib.MXMatrix(M.codes.to(torch.int8), M.scales, 40, lib.CODED_MX4)
    f = torch.zeros
    for X, Y, more in [(f(41, 2), f(6, 2), {}), (f(40, 2), f(2, 6), {}), (f(40, 2, dtype=torch.float64), f(6, 2), {"x": 1}),
                       (f(40, 2).int(), f(6, 2), {}), (f(2, 40).t(), f(6, 2), {}), (f(40, 2), f(6, 2), dict(beta=1.0)),
                       (f(40, 2), f(6, 2), dict(beta=1.0, C=f(6, 2, dtype=torch.bfloat16))), (f(40, 2), f(6, 2), dict(beta=1.0, C=f(6))),
                       (f(40, 2, 1), f(6, 2), {}), (M, f(6, 6), {}), (f(2, 41), f(6, 2), dict(x_rows=True))]:
        with pytest.raises((ValueError, lib.CodedError)):
            lib.coded_mx_mm(M, X, Y, **{k: v for k, v in more.items() if k != "x"})
    with pytest.raises(ValueError):
        lib.coded_mx_mm_t(M, M, f(40, 6), x_rows=True)
    with pytest.raises(ValueError):
        lib.coded_mx_quantize(f(6, 41), M)
    with pytest.raises(ValueError):
        lib.coded_mx_dequantize(M, f(5, 40))


@pytest.mark.parametrize("transposed", [False, True])
def test_workspace_of_a_call_on_a_stream_is_that_streams(lib, monkeypatch, transposed):
    """Memory handed out for the current stream may still be read or written by work that waits there, which a kernel
    on another stream does not wait for: the automatic workspace is asked for with the call's stream as the current one."""
    torch = pytest.importorskip("torch")
    q, r, s = (100000, 512, 2) if transposed else (512, 40000, 9)
    assert lib.coded_mx_workspace(transposed, lib.CODED_MX4, q, r, lib.CODED_F32, s) > 0
    M = lib.alloc_mx(q, r, lib.CODED_MX4, device="cpu")
    k, n = (q, r) if transposed else (r, q)
    X, Y = torch.empty((k, s)), torch.empty((n, s))

    class Buffer:
        def data_ptr(self):
            return 0x1000

        def record_stream(self, stream):
            pass

    class Torch:
        uint8 = torch.uint8
        current = None
        asked = []

        def empty(self, *a, **k):
            self.asked.append(self.current)
            return Buffer()

        @property
        def cuda(self):
            outer = self

            class Cuda:
                @staticmethod
                @contextlib.contextmanager
                def stream(s):
                    outer.current, before = s, outer.current
                    yield
                    outer.current = before
            return Cuda

    real = lib.lib()

    class Library:
        coded_mx_workspace = real.coded_mx_workspace

        def __getattr__(self, name):
            return lambda *a: lib.CODED_OK

    fake, side = Torch(), types.SimpleNamespace(cuda_stream=7)
    lib._dtype_code(X)
    monkeypatch.setattr(lib, "_torch", lambda: fake)
    monkeypatch.setattr(lib, "lib", Library)
    (lib.coded_mx_mm_t if transposed else lib.coded_mx_mm)(M, X, Y, stream=side)
    assert fake.asked == [side] and fake.current is None


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("change", [dict(alpha=1e300), dict(alpha=-3.5e38), dict(beta=1e39, C=0x5000, ldcc=2), dict(beta=-1e300, C=0x5000, ldcc=2)])
def test_alpha_and_beta_that_are_no_fp32_numbers_are_refused(lib, transposed, change):
    """They enter in fp32, where these would be infinite."""
    assert _call(lib, transposed, **change) == lib.CODED_ERR_ARG
    assert "alpha and beta" in lib.last_error()


@pytest.mark.parametrize("transposed", [False, True])
def test_alpha_and_beta_of_the_largest_fp32_number_pass(lib, transposed):
    top = float(np.finfo(np.float32).max)
    assert _call(lib, transposed, s=0, alpha=top, beta=-top, C=0x5000, ldcc=2) == lib.CODED_OK


@pytest.mark.parametrize("sizes", [(2 ** 41, 64, 1), (64, 2 ** 41, 1), (64, 64, 2 ** 41), (64, 64, 2 ** 62), (2 ** 62, 2 ** 62, 2 ** 62)])
@pytest.mark.parametrize("transposed", [0, 1])
def test_workspace_of_sizes_that_no_call_takes_is_refused(lib, transposed, sizes):
    b = ctypes.c_int64()
    q, r, s = sizes
    assert lib.lib().coded_mx_workspace(transposed, 3, q, r, 0, s, 0, ctypes.addressof(b)) == lib.CODED_ERR_SHAPE
    assert lib.last_error()
