"""Microscaled matrices on the GPU against the oracle in 64 bits.

Bounds.  A term of a product (code times scale times an element of X, or a
third of it) is exact in fp32, so a result differs from the exact sum by the
roundings of fp32 additions alone: with k terms, however they are ordered and
whether additions round or cut off, by less than terms * 2^-23 times the sum of
the magnitudes (terms: 3 k for an fp32 X, which enters as three numbers), plus
2^-22 of the result and of beta C for the epilogue, plus half a bf16 step
(2^-8 of the result) where the result is bf16.  Whole numbers small enough are exact.
"""
import math

import numpy as np
import pytest

from oracle import mx as om
from tests.gpu_helpers import torch_mod

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    t = torch_mod()
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    return t


def fmt_of(lib, bits):
    return lib.CODED_MX4 if bits == 4 else lib.CODED_MX8


def microscaled(lib, torch, rng, rows, cols, bits, pad=0, whole=False):
    """(MXMatrix, fp64 values).  whole: scales of 1 and whole codes.  pad: 16-byte pieces and 4-byte
    words of 0xFF behind each row."""
    blocks = -(-cols // 32)
    if whole:
        table = om.format_values(bits)
        pick = [c for c, v in enumerate(table) if v == round(v) and abs(v) <= 6] if bits == 4 else \
            [c for c, v in enumerate(table) if np.isfinite(v) and v == round(v) and abs(v) <= 8]
        codes = np.array(pick, dtype=np.uint8)[rng.integers(0, len(pick), (rows, blocks * 32))]
        scales = np.full((rows, blocks), 127, dtype=np.uint8)
    else:
        codes = rng.integers(0, 16 if bits == 4 else 256, (rows, blocks * 32)).astype(np.uint8)
        if bits == 8:
            codes[(codes & 0x7F) == 0x7F] = 0x7E
        scales = rng.integers(120, 126, (rows, blocks)).astype(np.uint8)
    codes[:, cols:] = 0
    v = om.values(codes, scales, cols, bits)
    c, s = om.pack(codes, scales, bits)
    c = np.concatenate([c, np.full((rows, 16 * pad), 0xFF, np.uint8)], 1)
    s = np.concatenate([s, np.full((rows, 4 * pad), 0xFF, np.uint8)], 1)
    return lib.MXMatrix(torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda(), cols, fmt_of(lib, bits)), v


def dense(torch, a, dtype, pad=0):
    """a on the device, in rows `pad` elements further apart, NaN between them."""
    wide = np.full((a.shape[0], a.shape[1] + pad), np.nan, np.float32)
    wide[:, :a.shape[1]] = a
    return torch.from_numpy(wide).cuda().to(dtype)[:, :a.shape[1]]


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


def check_product(lib, torch, rng, transposed, q, r, s, bits, x, y, x_rows, y_rows, pad=0, alpha=1.0, beta=0.0, whole=False):
    M, A = microscaled(lib, torch, rng, q, r, bits, pad, whole)
    k, n = (q, r) if transposed else (r, q)
    if x.startswith("mx"):
        X, xv = microscaled(lib, torch, rng, s, k, int(x[2:]), pad, whole)
        xv = xv.T
    else:
        xv = rng.integers(-7, 8, (k, s)).astype(np.float64) if whole else rng.standard_normal((k, s)) * rng.choice([0.01, 1, 30], (1, s))
        xv = xv.astype(np.float32)
        if x == "bf16":
            xv = torch.from_numpy(xv).bfloat16().float().numpy()
        X = dense(torch, xv.T if x_rows else xv, torch.bfloat16 if x == "bf16" else torch.float32, pad)
        xv = xv.astype(np.float64)
    dt = torch.bfloat16 if y == "bf16" else torch.float32
    shape = (s, n) if y_rows else (n, s)
    wide = torch.full((shape[0] + 2, shape[1] + pad), 7.0, dtype=dt, device="cuda")
    Y = wide[1:-1, :shape[1]]
    cv, C = 0.0, None
    if beta:
        cv = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(dt).float().numpy().astype(np.float64)
        C = dense(torch, cv, dt, pad)
    A_ = A.T if transposed else A
    if whole:      # exact in 64 bits wherever it is computed
        want = size = (torch.from_numpy(np.ascontiguousarray(A_)).cuda() @ torch.from_numpy(np.ascontiguousarray(xv)).cuda()).cpu().numpy()
    else:
        want, size = A_ @ xv, np.abs(A_) @ np.abs(xv)
    if y_rows:
        want, size = want.T, size.T
    want, size = alpha * want + beta * cv, abs(alpha) * size
    (lib.coded_mx_mm_t if transposed else lib.coded_mx_mm)(M, X, Y, x_rows=x_rows, y_rows=y_rows, alpha=alpha, beta=beta, C=C)
    torch.cuda.synchronize()
    got = host(Y)
    if whole:
        assert np.array_equal(got, want)
    else:
        bound = (3 if x == "f32" else 1) * k * 2.0 ** -23 * size + 2.0 ** -22 * (np.abs(want) + np.abs(beta * cv)) + 2.0 ** -120
        if y == "bf16":
            bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
        assert np.all(np.abs(got - want) <= bound), np.max(np.abs(got - want) / bound)
    # nothing around the result is touched
    assert bool((wide[0] == 7).all()) and bool((wide[-1] == 7).all()) and bool((wide[:, shape[1]:] == 7).all())


# ---------------------------------------------------------------- storing

@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("q,r,pad", [(1, 1, 0), (3, 31, 1), (7, 32, 0), (5, 33, 3), (300, 4, 0), (9, 127, 5), (4, 128, 0), (2, 2049, 1), (17, 5750, 0)])
def test_stored_codes_equal_the_oracles(lib, torch, bits, dtype, q, r, pad):
    rng = np.random.default_rng(q * 10007 + r * 11 + bits)
    a = (rng.standard_normal((q, r)) * 2.0 ** rng.integers(-20, 20, (q, r))).astype(np.float32)
    a[rng.random((q, r)) < 0.3] *= 0
    near = rng.random((q, r)) < 0.3        # ties and the edges of the formats
    a[near] = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7, 7.99, 448, 464, 465, 500, 2.0 ** -10, 3 * 2.0 ** -10, -0.0], near.sum())
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    A = dense(torch, a, dt, pad)
    av = host(A)
    M = lib.alloc_mx(q, r, fmt_of(lib, bits))
    wide_c = torch.full((q, M.codes.shape[1] + 16 * pad), 0xAB, dtype=torch.uint8, device="cuda")
    wide_s = torch.full((q, M.scales.shape[1] + 4 * pad), 0xAB, dtype=torch.uint8, device="cuda")
    M = lib.MXMatrix(wide_c, wide_s, r, M.fmt)
    lib.coded_mx_quantize(A, M)
    codes, scales = om.quantize(av, bits)
    want_c, want_s = om.pack(codes, scales, bits)
    assert np.array_equal(wide_s.cpu().numpy()[:, :want_s.shape[1]], want_s)
    assert np.array_equal(wide_c.cpu().numpy()[:, :want_c.shape[1]], want_c)
    assert bool((wide_c[:, want_c.shape[1]:] == 0xAB).all()) and bool((wide_s[:, want_s.shape[1]:] == 0xAB).all())
    for out_dt in (torch.float32, torch.bfloat16):
        out = torch.full((q, r + pad), 7.0, dtype=out_dt, device="cuda")
        lib.coded_mx_dequantize(M, out[:, :r])
        assert np.array_equal(host(out[:, :r]), om.values(codes, scales, r, bits))
        assert bool((out[:, r:] == 7).all())


@pytest.mark.parametrize("bits", [4, 8])
def test_blocks_that_hold_no_numbers_or_nothing(lib, torch, bits):
    a = np.ones((6, 96), np.float32)
    a[0, 40] = np.inf
    a[1, 0] = np.nan
    a[2, 95] = -np.inf
    a[3, 32:64] = 0
    a[4, :32] = 1e-45
    a[5, 64:] = 3.4028234e38
    M = lib.alloc_mx(6, 96, fmt_of(lib, bits))
    lib.coded_mx_quantize(torch.from_numpy(a).cuda(), M)
    codes, scales = om.quantize(a.astype(np.float64), bits)
    assert np.array_equal(M.scales.cpu().numpy()[:, :3], scales)
    assert np.array_equal(M.codes.cpu().numpy(), om.pack(codes, scales, bits)[0])
    assert list(scales[0]) == [scales[0, 0], 255, scales[0, 0]] and scales[3, 1] == 10 and scales[4, 0] == 10
    out = torch.empty((6, 96), dtype=torch.float32, device="cuda")
    lib.coded_mx_dequantize(M, out)
    assert np.array_equal(host(out), om.values(codes, scales, 96, bits), equal_nan=True)


def test_a_saved_batch_saves_the_same_again(lib, torch):
    """Codes of values that are in the format already are those values (the cut-down maximum included)."""
    g = torch.Generator(device="cuda").manual_seed(5)
    a = torch.randn((333, 1000), generator=g, device="cuda")
    for fmt in (lib.CODED_MX4, lib.CODED_MX8):
        M, N = lib.alloc_mx(333, 1000, fmt), lib.alloc_mx(333, 1000, fmt)
        b = torch.empty_like(a)
        lib.coded_mx_quantize(a, M)
        lib.coded_mx_dequantize(M, b)
        lib.coded_mx_quantize(b, N)
        c = torch.empty_like(a)
        lib.coded_mx_dequantize(N, c)
        assert torch.equal(b, c)


# ---------------------------------------------------------------- products

TERMS = [1, 31, 33, 128, 300, 2050]
SHAPES = [(1, 1), (17, 1), (1, 17), (15, 2), (16, 5), (130, 16), (65, 17), (64, 64), (130, 65), (300, 129)]


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("k", TERMS)
def test_products(lib, torch, transposed, bits, x, k):
    rng = np.random.default_rng(k * 17 + bits + 100 * transposed)
    for at, (n, s) in enumerate(SHAPES):
        q, r = (k, n) if transposed else (n, k)
        check_product(lib, torch, rng, transposed, q, r, s, bits, x, ["f32", "bf16"][at % 2], bool(at & 1), bool(at & 2),
                      pad=at % 3, alpha=[1.0, -0.5][at % 2], beta=[0.0, 1.0, -2.0][at % 3])


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("x_rows", [False, True])
@pytest.mark.parametrize("y_rows", [False, True])
@pytest.mark.parametrize("y", ["f32", "bf16"])
def test_every_order_and_type(lib, torch, transposed, x, x_rows, y_rows, y):
    rng = np.random.default_rng(3)
    for bits, n, k, s, pad in [(4, 200, 96, 1, 0), (8, 70, 100, 3, 1), (4, 257, 513, 40, 8), (8, 260, 320, 300, 0), (4, 600, 64, 260, 1)]:
        q, r = (k, n) if transposed else (n, k)
        check_product(lib, torch, rng, transposed, q, r, s, bits, x, y, x_rows, y_rows, pad=pad, alpha=2.0, beta=0.5)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("x", ["mx4", "mx8"])
@pytest.mark.parametrize("k", TERMS)
def test_products_of_two_microscaled(lib, torch, bits, x, k):
    rng = np.random.default_rng(k * 19 + bits)
    for at, (n, s) in enumerate(SHAPES + [(520, 300)]):
        check_product(lib, torch, rng, False, n, k, s, bits, x, ["f32", "bf16"][at % 2], True, bool(at & 2), pad=at % 3,
                      alpha=[1.0, -0.5][at % 2], beta=[0.0, 1.0, -2.0][at % 3])


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("x", ["f32", "bf16", "mx4", "mx8"])
def test_whole_numbers_are_exact(lib, torch, transposed, bits, x):
    """Sums of whole numbers below 2^24 have one right answer."""
    if transposed and x.startswith("mx"):
        pytest.skip("U is dense")
    rng = np.random.default_rng(11)
    for n, k, s in [(1, 1, 1), (40, 77, 1), (100, 1000, 3), (513, 4100, 1), (300, 640, 16), (33, 2500, 64), (256, 256, 256), (290, 1111, 270)]:
        q, r = (k, n) if transposed else (n, k)
        for order in range(4):
            if x.startswith("mx") and not order & 1:
                continue
            check_product(lib, torch, rng, transposed, q, r, s, bits, x, "f32", bool(order & 1), bool(order & 2), whole=True)


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("x", ["f32", "bf16", "mx4", "mx8"])
def test_whole_numbers_are_exact_in_large_tiles_and_long_sums(lib, torch, transposed, bits, x):
    if transposed and x.startswith("mx"):
        pytest.skip("U is dense")
    rng = np.random.default_rng(13)
    for n, k, s, order in [(8190, 130, 1030, 3), (8193, 8300, 1025, 1), (8193, 200, 1027, 0), (40, 20000, 100, 1), (300, 9000, 200, 3)]:
        q, r = (k, n) if transposed else (n, k)
        check_product(lib, torch, rng, transposed, q, r, s, bits, x, "f32", bool(order & 1) or x.startswith("mx"), bool(order & 2), whole=True,
                      alpha=-1.0, beta=0.0)


@pytest.mark.parametrize("transposed", [False, True])
def test_every_bit_of_an_fp32_x_counts(lib, torch, transposed):
    """One code of 1 in each sum: the result is X's element itself."""
    rng = np.random.default_rng(8)
    k, n = 96, 96
    for s in (1, 4, 7, 33, 200):
        codes = np.zeros((k, n), np.uint8)
        codes[np.arange(k), rng.permutation(n)] = 2
        cs, ss = om.pack(codes, np.full((k, n // 32), 127, np.uint8), 4)
        M = lib.MXMatrix(torch.from_numpy(cs).cuda(), torch.from_numpy(ss).cuda(), n, lib.CODED_MX4)
        X = (rng.standard_normal((k, s)) * 10.0 ** rng.integers(-20, 20, (k, s))).astype(np.float32)
        X[0, 0], X[1, 0] = 3.4028235e38, -1.1754944e-38
        P = om.values(codes, np.full((k, n // 32), 127, np.uint8), n, 4)
        Y = torch.empty((n, s), device="cuda")
        (lib.coded_mx_mm_t if transposed else lib.coded_mx_mm)(M, torch.from_numpy(X).cuda(), Y)
        # a value's lowest piece may fall below the smallest bf16 number, 2^-133
        assert np.all(np.abs(host(Y) - ((P.T if transposed else P) @ X.astype(np.float64))) <= 2.0 ** -131)


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("s", [1, 5, 40, 200])
@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_no_terms(lib, torch, transposed, s, x):
    n = 70
    M = lib.alloc_mx(0 if transposed else n, n if transposed else 0, lib.CODED_MX4)
    X = torch.empty((0, s), device="cuda", dtype=torch.float32 if x == "f32" else torch.bfloat16)
    Y = torch.full((n, s), 7.0, device="cuda")
    C = torch.randn((n, s), device="cuda")
    call = lib.coded_mx_mm_t if transposed else lib.coded_mx_mm
    call(M, X, Y)
    assert bool((Y == 0).all())
    call(M, X, Y, beta=-2.0, C=C)
    assert torch.equal(Y, -2.0 * C)


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("x", ["f32", "bf16", "mx4"])
@pytest.mark.parametrize("n,k,s", [(40, 70, 1), (40, 70, 3), (140, 330, 20), (300, 200, 200)])
def test_no_number_spreads_no_further_than_its_sums(lib, torch, transposed, bits, x, n, k, s):
    if transposed and x == "mx4":
        pytest.skip("U is dense")
    rng = np.random.default_rng(21)
    q, r = (k, n) if transposed else (n, k)
    M, A = microscaled(lib, torch, rng, q, r, bits, pad=1)
    M.scales[q // 2, (r - 1) // 32] = 255           # the row's last block, which r ends inside of
    b0 = (r - 1) // 32 * 32
    A[q // 2, b0:] = np.nan
    if x == "mx4":
        X, xv = microscaled(lib, torch, rng, s, k, 4)
        X.scales[s - 1, 0] = 255
        xv[s - 1, :32] = np.nan
        xv = xv.T
    else:
        xv = rng.standard_normal((k, s)).astype(np.float32)
        xv[k - 1, s - 1] = np.inf
        X = dense(torch, xv, torch.bfloat16 if x == "bf16" else torch.float32, 3)
        xv = host(X)
    Y = torch.empty((n, s), device="cuda")
    (lib.coded_mx_mm_t if transposed else lib.coded_mx_mm)(M, X, Y, x_rows=x == "mx4")
    A_ = A.T if transposed else A
    with np.errstate(invalid="ignore"):
        want = np.stack([np.stack([np.sum(A_[i] * xv[:, c]) for c in range(s)]) for i in range(n)])
    got = host(Y)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]) and np.all(np.isfinite(got[np.isfinite(want)]))


def test_c_of_one_row_and_in_place(lib, torch):
    rng = np.random.default_rng(4)
    M, A = microscaled(lib, torch, rng, 90, 70, 4, whole=True)
    x = rng.integers(-5, 6, (11, 70)).astype(np.float32)
    bias = rng.integers(-9, 10, 90).astype(np.float32)
    Y = torch.empty((11, 90), device="cuda")
    lib.coded_mx_mm(M, torch.from_numpy(x).cuda(), Y, x_rows=True, y_rows=True, beta=1.0, C=torch.from_numpy(bias).cuda())
    assert np.array_equal(host(Y), x @ A.T + bias)
    lib.coded_mx_mm(M, torch.from_numpy(x).cuda(), Y, x_rows=True, y_rows=True, alpha=-2.0, beta=1.0, C=Y)
    assert np.array_equal(host(Y), -(x @ A.T) + bias)


def test_vectors_and_tensors_of_one_row(lib, torch):
    rng = np.random.default_rng(6)
    M, A = microscaled(lib, torch, rng, 50, 64, 4, whole=True)
    x = rng.integers(-5, 6, 64).astype(np.float32)
    X = torch.from_numpy(x).cuda()
    for xs, x_rows in ((X, False), (X, True), (X[:, None], False), (X[None], True), (X[None].t(), False), (X[:, None].t(), True)):
        for ys, y_rows in ((torch.empty(50), False), (torch.empty(50), True), (torch.empty(50, 1), False), (torch.empty(1, 50), True)):
            ys = ys.cuda()
            lib.coded_mx_mm(M, xs, ys, x_rows=x_rows, y_rows=y_rows)
            assert np.array_equal(host(ys).reshape(-1), A @ x)


@pytest.mark.parametrize("transposed", [False, True])
def test_same_bits_every_time_and_on_another_stream(lib, torch, transposed):
    rng = np.random.default_rng(9)
    for n, k, s in [(300, 5000, 1), (300, 5000, 8), (700, 900, 300)]:
        q, r = (k, n) if transposed else (n, k)
        M, _ = microscaled(lib, torch, rng, q, r, 4)
        X = torch.randn((k, s), device="cuda")
        call = lib.coded_mx_mm_t if transposed else lib.coded_mx_mm
        Y = [torch.empty((n, s), device="cuda") for _ in range(3)]
        call(M, X, Y[0])
        call(M, X, Y[1])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        call(M, X, Y[2], stream=side)
        side.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(Y[0], Y[1]) and torch.equal(Y[0], Y[2])


@pytest.mark.parametrize("transposed", [False, True])
def test_captured_and_replayed(lib, torch, transposed):
    rng = np.random.default_rng(10)
    n, k, s = 500, 3000, 4
    q, r = (k, n) if transposed else (n, k)
    M, A = microscaled(lib, torch, rng, q, r, 4, whole=True)
    A = A.T if transposed else A
    X = torch.zeros((k, s), device="cuda")
    Y = torch.empty((n, s), device="cuda")
    call = lib.coded_mx_mm_t if transposed else lib.coded_mx_mm
    wsb = lib.coded_mx_workspace(transposed, M.fmt, q, r, lib.CODED_F32, s)
    ws = torch.empty(max(wsb, 16), dtype=torch.uint8, device="cuda")
    call(M, X, Y, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(M, X, Y, workspace=ws)
    for i in range(4):
        x = rng.integers(-5, 6, (k, s)).astype(np.float32)
        X.copy_(torch.from_numpy(x))
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(host(Y), A @ x), i


def test_rows_past_4_gib(lib, torch):
    """Codes longer than 2^32 bytes: the last rows' products equal those of the same rows by themselves."""
    q, r = (1 << 19) + 77, 16384
    codes = torch.randint(0, 256, (q, r // 2), dtype=torch.uint8, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    assert codes.numel() > 1 << 32
    scales = torch.full((q, r // 32), 127, dtype=torch.uint8, device="cuda")
    M = lib.MXMatrix(codes, scales, r, lib.CODED_MX4)
    tail = M.rows(q - 200, q)
    g = torch.Generator(device="cuda").manual_seed(2)
    for s in (1, 20):
        X = torch.randint(-3, 4, (r, s), device="cuda", generator=g).bfloat16()
        Y, T = torch.empty((q, s), device="cuda"), torch.empty((200, s), device="cuda")
        lib.coded_mx_mm(M, X, Y)
        lib.coded_mx_mm(tail, X, T)
        assert torch.equal(Y[q - 200:], T)
        U = torch.zeros((q, s), device="cuda", dtype=torch.bfloat16)
        U[q - 200:] = torch.randint(-3, 4, (200, s), device="cuda", generator=g).bfloat16()
        Z, V = torch.empty((r, s), device="cuda"), torch.empty((r, s), device="cuda")
        lib.coded_mx_mm_t(M, U, Z)
        lib.coded_mx_mm_t(tail, U[q - 200:].contiguous(), V)
        assert torch.equal(Z, V)   # whole numbers below 2^24: exact


def test_gradients_against_differences(lib, torch):
    """loss = |X W^T + b - T|^2 / 2 over a saved batch X: the gradients the products give against central
    differences of the loss in 64 bits (quadratic: differences are exact but for rounding)."""
    rng = np.random.default_rng(12)
    tokens, fan_in, fan_out = 24, 70, 50
    W, Wv = microscaled(lib, torch, rng, fan_out, fan_in, 4)
    Xs, Xv = microscaled(lib, torch, rng, tokens, fan_in, 8)
    T = rng.standard_normal((tokens, fan_out)).astype(np.float32)
    D = torch.empty((tokens, fan_out), device="cuda")
    lib.coded_mx_mm(W, Xs, D, x_rows=True, y_rows=True, beta=-1.0, C=torch.from_numpy(T).cuda())
    dX = torch.empty((tokens, fan_in), device="cuda")
    lib.coded_mx_mm_t(W, D, dX, x_rows=True, y_rows=True)
    dW = torch.empty((fan_out, fan_in), device="cuda")
    lib.coded_mx_mm_t(Xs, D, dW, y_rows=True)

    def loss(x, w):
        return 0.5 * np.sum((x @ w.T - T) ** 2)

    got_x, got_w = host(dX), host(dW)
    for _ in range(12):
        e = rng.standard_normal(Xv.shape)
        num = (loss(Xv + 1e-3 * e, Wv) - loss(Xv - 1e-3 * e, Wv)) / 2e-3
        assert abs(num - np.sum(got_x * e)) <= 1e-5 * np.sum(np.abs(got_x * e))
        e = rng.standard_normal(Wv.shape)
        num = (loss(Xv, Wv + 1e-3 * e) - loss(Xv, Wv - 1e-3 * e)) / 2e-3
        assert abs(num - np.sum(got_w * e)) <= 1e-5 * np.sum(np.abs(got_w * e))
    d = Xv @ Wv.T - T
    assert np.allclose(got_x, d @ Wv, rtol=1e-4, atol=1e-4 * np.max(np.abs(got_x)))
    assert np.allclose(got_w, d.T @ Xv, rtol=1e-4, atol=1e-4 * np.max(np.abs(got_w)))


def test_workspace_too_small_is_refused(lib, torch):
    need = lib.coded_mx_workspace(True, lib.CODED_MX4, 100000, 512, lib.CODED_F32, 1)
    if need == 0:
        pytest.skip("no workspace for these sizes")
    M = lib.alloc_mx(100000, 512, lib.CODED_MX4)
    with pytest.raises(lib.CodedError) as e:
        lib.coded_mx_mm_t(M, torch.zeros(100000, device="cuda"), torch.zeros(512, device="cuda"),
                          workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    assert e.value.status == lib.CODED_ERR_ARG
    assert math.isfinite(need)


def whole_codes(torch, rows, cols, g):
    """Codes of whole numbers up to 6 (4 bits) with scales of 1, made on the GPU, and the fp64 values."""
    table = torch.tensor([0, 2, 4, 5, 6, 7, 10, 12, 13, 14, 15], device="cuda", dtype=torch.uint8)
    pick = torch.randint(0, len(table), (rows, -(-cols // 32) * 32), device="cuda", generator=g)
    codes = table[pick]
    codes[:, cols:] = 0
    value = torch.tensor(om.format_values(4), device="cuda")
    v = value[codes.int()][:, :cols]
    packed = codes[:, 0::2] | (codes[:, 1::2] << 4)
    return packed.contiguous(), torch.full((rows, -(-cols // 128) * 4), 127, dtype=torch.uint8, device="cuda"), v


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("x", ["f32", "bf16", "mx4"])
@pytest.mark.parametrize("n,k,s", [(8192, 16500, 2048), (8448, 200, 2100), (520, 66000, 260)])
def test_whole_numbers_are_exact_over_rounds_of_tiles(lib, torch, transposed, x, n, k, s):
    """More than a round of large tiles with some left over, sums of more than one fp32 chain, and sums split many times."""
    if transposed and x == "mx4":
        pytest.skip("U is dense")
    g = torch.Generator(device="cuda").manual_seed(n + k + s)
    q, r = (k, n) if transposed else (n, k)
    codes, scales, A = whole_codes(torch, q, r, g)
    M = lib.MXMatrix(codes, scales, r, lib.CODED_MX4)
    A = A.t() if transposed else A
    for order in (0, 3):
        if x == "mx4":
            xc, xs, X64 = whole_codes(torch, s, k, g)
            X, X64 = lib.MXMatrix(xc, xs, k, lib.CODED_MX4), X64.t()
        else:
            X = torch.randint(-7, 8, (s, k) if order & 1 else (k, s), device="cuda", generator=g).to(torch.float32 if x == "f32" else torch.bfloat16)
            X64 = X.double().t() if order & 1 else X.double()
        Y = torch.empty((s, n) if order & 2 else (n, s), device="cuda")
        (lib.coded_mx_mm_t if transposed else lib.coded_mx_mm)(M, X, Y, x_rows=bool(order & 1) or x == "mx4", y_rows=bool(order & 2))
        want = A @ X64
        assert float(want.abs().max()) < 2 ** 24
        assert torch.equal(Y.double(), want.t() if order & 2 else want)


@pytest.mark.parametrize("transposed", [False, True])
def test_x_by_columns_at_any_address(lib, torch, transposed):
    """Columns of bf16 at even and odd row strides and addresses: read as they are, or copied."""
    g = torch.Generator(device="cuda").manual_seed(3)
    for n, k, s in ((700, 300, 130), (8200, 130, 1100)):
        q, r = (k, n) if transposed else (n, k)
        codes, scales, A = whole_codes(torch, q, r, g)
        M = lib.MXMatrix(codes, scales, r, lib.CODED_MX4)
        A = A.t() if transposed else A
        for ld, off in ((s, 0), (s + 1, 0), (s + 2, 1), (s + 2, 2), (s + 7, 3)):
            flat = torch.full((k * ld + off + 8,), float("nan"), dtype=torch.bfloat16, device="cuda")
            X = flat[off:off + k * ld].view(k, ld)[:, :s]
            X.copy_(torch.randint(-7, 8, (k, s), device="cuda", generator=g))
            Y = torch.empty((n, s), device="cuda")
            (lib.coded_mx_mm_t if transposed else lib.coded_mx_mm)(M, X, Y)
            assert torch.equal(Y.double(), A @ X.double()), (ld, off)


def test_rows_of_more_than_eight_megabytes(lib, torch):
    """Offsets within a tile's rows that pass 32 bits take the general kernel."""
    r = (1 << 24) + 5
    g = torch.Generator(device="cuda").manual_seed(4)
    codes, scales, A = whole_codes(torch, 2, r, g)
    codes[:, 1 << 18:] = 0          # sums below 2^24
    A[:, 1 << 19:] = 0
    M = lib.MXMatrix(codes, scales, r, lib.CODED_MX4)
    X = torch.randint(-7, 8, (r, 2), device="cuda", generator=g).to(torch.bfloat16)
    Y = torch.empty((2, 2), device="cuda")
    lib.coded_mx_mm(M, X, Y)
    assert torch.equal(Y.double(), A @ X.double())
    U = torch.tensor([[1.0, 2.0], [3.0, -1.0]], device="cuda")
    Z = torch.empty((r, 2), device="cuda")
    lib.coded_mx_mm_t(M, U, Z)
    assert torch.equal(Z.double(), A.t() @ U.double())


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("x", ["f32", "bf16", "mx4", "mx8"])
def test_one_vector_and_long_rows(lib, torch, bits, x):
    rng = np.random.default_rng(31)
    for q, r, order, whole in [(4096, 2048, 3, True), (4099, 2050, 1, False), (20485, 2081, 0, True), (4103, 16384, 3, True), (4130, 16417, 2, True),
                               (4097, 33001, 1, True)]:
        check_product(lib, torch, rng, False, q, r, 1, bits, x, "bf16" if order == 1 and not whole else "f32", bool(order & 1) or x.startswith("mx"),
                      bool(order & 2), pad=order, alpha=-1.0, beta=0.0 if whole else 0.5, whole=whole)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("r", [2050, 18000])
def test_no_number_in_a_long_row_spreads_to_no_other(lib, torch, bits, r):
    rng = np.random.default_rng(33)
    q = 4100
    M, A = microscaled(lib, torch, rng, q, r, bits)
    M.scales[77, (r - 1) // 32] = 255
    M.scales[q - 1, 0] = 255
    x = torch.randn(r, device="cuda")
    Y = torch.empty(q, device="cuda")
    lib.coded_mx_mm(M, x, Y)
    bad = np.isnan(host(Y))
    assert bad.sum() == 2 and bad[77] and bad[q - 1]
    x[r - 1] = float("inf")
    lib.coded_mx_mm(M, x, Y)
    last = A[:, r - 1].copy()
    last[[77, q - 1]] = 0.0          # 0 times an infinity, like NaN times it, is NaN
    got = host(Y)
    assert np.array_equal(np.isnan(got), last == 0) and np.array_equal(got[last != 0], np.copysign(np.inf, last[last != 0]))


@pytest.mark.parametrize("q,r", [(4100, 4100), (4099, 8190), (262144, 2050), (32768, 16390), (33001, 16384)])
def test_one_vector_however_it_lies(lib, torch, q, r):
    """fp32 and bf16, contiguous, at every bf16 address, and strided; matrices below and above 256 MB."""
    g = torch.Generator(device="cuda").manual_seed(6)
    codes, scales, A = whole_codes(torch, q, r, g)
    M = lib.MXMatrix(codes, scales, r, lib.CODED_MX4)
    for dtype in (torch.float32, torch.bfloat16):
        for off, step in ((0, 1), (1, 1), (2, 1), (3, 2)):
            flat = torch.full((off + r * step + 8,), float("nan"), dtype=dtype, device="cuda")
            X = flat[off:off + r * step].view(r, step)[:, :1]
            X.copy_(torch.randint(-7, 8, (r, 1), device="cuda", generator=g))
            wide = torch.full((q + 2, 1), 7.0, device="cuda")
            lib.coded_mx_mm(M, X, wide[1:-1])
            assert torch.equal(wide[1:-1].double(), A @ X.double()), (dtype, off, step)
            assert wide[0] == 7 and wide[-1] == 7


def whole_codes_of(torch, bits, rows, cols, g):
    """whole_codes in 4 or 8 bits (whole numbers up to 8 there)."""
    if bits == 4:
        return whole_codes(torch, rows, cols, g)
    values = om.format_values(8)
    table = torch.tensor([c for c, v in enumerate(values) if np.isfinite(v) and v == round(v) and abs(v) <= 8], device="cuda", dtype=torch.uint8)
    codes = table[torch.randint(0, len(table), (rows, -(-cols // 32) * 32), device="cuda", generator=g)]
    codes[:, cols:] = 0
    v = torch.tensor(values, device="cuda")[codes.int()][:, :cols]
    return codes, torch.full((rows, -(-cols // 128) * 4), 127, dtype=torch.uint8, device="cuda"), v


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("bits", [4, 8])
def test_an_odd_number_of_columns_of_x_in_even_rows(lib, torch, transposed, bits):
    """bf16 columns that are read as they are: with s odd the last row's last word holds the last side's term and
    nothing else of X.  That row is made of numbers that every last side's result shows."""
    g = torch.Generator(device="cuda").manual_seed(5)
    for n, k, s in ((300, 1, 67), (700, 300, 131), (90, 3, 67), (260, 64, 65), (8200, 130, 1101), (130, 65, 8191), (8200, 128, 1027), (8200, 130, 2047)):
        q, r = (k, n) if transposed else (n, k)
        codes, scales, A = whole_codes_of(torch, bits, q, r, g)
        M = lib.MXMatrix(codes, scales, r, fmt_of(lib, bits))
        A = A.t() if transposed else A
        for ld, off in ((s + 1, 0), (s + 1, 2), (s + 7, 4)):
            flat = torch.full((off + (k - 1) * ld + s,), float("nan"), dtype=torch.bfloat16, device="cuda")
            X = flat[off:].as_strided((k, s), (ld, 1))
            X.copy_(torch.randint(-7, 8, (k, s), device="cuda", generator=g))
            X[k - 1].fill_(9)
            for y_rows in (False, True):
                Y = torch.empty((s, n) if y_rows else (n, s), device="cuda")
                (lib.coded_mx_mm_t if transposed else lib.coded_mx_mm)(M, X, Y, y_rows=y_rows)
                want = A @ X.double()
                assert torch.equal(Y.double(), want.t() if y_rows else want), (n, k, s, ld, off, y_rows)


@pytest.mark.parametrize("transposed", [False, True])
def test_workspace_on_another_stream_leaves_the_current_ones_memory_alone(lib, torch, transposed):
    """A tensor that is let go of while work on the current stream has still to read it; a product on another stream
    whose workspace is as large comes meanwhile."""
    rng = np.random.default_rng(14)
    q, r, s = (60000, 512, 4) if transposed else (200, 40000, 9)
    M, A = microscaled(lib, torch, rng, q, r, 4, whole=True)
    A = A.T if transposed else A
    x = rng.integers(-5, 6, (A.shape[1], s)).astype(np.float32)
    X, Y = torch.from_numpy(x).cuda(), torch.empty((A.shape[0], s), device="cuda")
    call = lib.coded_mx_mm_t if transposed else lib.coded_mx_mm
    need = lib.coded_mx_workspace(transposed, M.fmt, q, r, lib.CODED_F32, s)
    assert need > 0
    side = torch.cuda.Stream()
    out = torch.zeros(need, dtype=torch.uint8, device="cuda")
    held = torch.full((need,), 7, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)     # some tens of milliseconds
    out.copy_(held)
    del held
    call(M, X, Y, stream=side)
    side.synchronize()
    assert np.array_equal(host(Y), A @ x)
    torch.cuda.synchronize()
    assert bool((out == 7).all())


@pytest.mark.parametrize("x_bits", [4, 8])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("far", ["codes", "scales"])
def test_microscaled_rows_of_x_eight_megabytes_apart(lib, torch, bits, x_bits, far):
    """Every so many rows of a long saved batch: the workspace of the query by sizes is enough at any pitch of X."""
    g = torch.Generator(device="cuda").manual_seed(15)
    n, k, s = 300, 200, 70
    codes, scales, A = whole_codes_of(torch, bits, n, k, g)
    M = lib.MXMatrix(codes, scales, k, fmt_of(lib, bits))
    xc, xs, X64 = whole_codes_of(torch, x_bits, s, k, g)
    wide = torch.empty((s, 1 << 23), dtype=torch.uint8, device="cuda")
    near = xc if far == "codes" else xs
    wide[:, :near.shape[1]] = near
    view = wide[:, :near.shape[1]]
    X = lib.MXMatrix(view if far == "codes" else xc, xs if far == "codes" else view, k, fmt_of(lib, x_bits))
    for y_rows in (False, True):
        Y = torch.empty((s, n) if y_rows else (n, s), device="cuda")
        lib.coded_mx_mm(M, X, Y, x_rows=True, y_rows=y_rows)
        want = A @ X64.t()
        assert torch.equal(Y.double(), want.t() if y_rows else want)


def dense_whole(torch, x, s, k, x_rows, g):
    """(X, its values s x k in 64 bits): whole numbers up to 7, or 4-bit codes of them (rows)."""
    if x == "mx4":
        c, e, v = whole_codes(torch, s, k, g)
        return (c, e), v
    X = torch.randint(-7, 8, (s, k) if x_rows else (k, s), device="cuda", generator=g).to(torch.float32 if x == "f32" else torch.bfloat16)
    return X, X.double() if x_rows else X.double().t()


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("x", ["f32", "bf16", "mx4"])
@pytest.mark.parametrize("n,k,s", [(8192, 16500, 2048), (8200, 33000, 2100), (520, 66000, 260)])
def test_long_sums_are_rounded_once_after_alpha_and_c(lib, torch, transposed, x, n, k, s):
    """Sums that are exact in fp32, of more than one chain, and a C that is far larger: alpha S + beta C in fp32 has one
    right answer.  C apart from Y, in Y itself, and as one row."""
    if transposed and x == "mx4":
        pytest.skip("U is dense")
    g = torch.Generator(device="cuda").manual_seed(n + k)
    q, r = (k, n) if transposed else (n, k)
    codes, scales, A = whole_codes(torch, q, r, g)
    M = lib.MXMatrix(codes, scales, r, lib.CODED_MX4)
    A = A.t() if transposed else A
    call = lib.coded_mx_mm_t if transposed else lib.coded_mx_mm
    X, X64 = dense_whole(torch, x, s, k, True, g)
    if x == "mx4":
        X = lib.MXMatrix(*X, k, lib.CODED_MX4)
    S = X64 @ A.t()
    del A, X64
    assert float(S.abs().max()) < 2 ** 23
    for y_rows in (True, False):
        want = S if y_rows else S.t()
        C = (torch.randint(-100, 101, want.shape, device="cuda", generator=g) * 2.0 ** 24 + 2.0 ** 20).float()
        Y = C.clone()
        call(M, X, Y, x_rows=True, y_rows=y_rows, alpha=-0.5, beta=1.0, C=Y)
        assert torch.equal(Y, (C.double() - 0.5 * want).float())
        call(M, X, Y, x_rows=True, y_rows=y_rows, alpha=2.0, beta=-1.0, C=C)
        assert torch.equal(Y, (2.0 * want - C.double()).float())
        call(M, X, Y, x_rows=True, y_rows=y_rows, alpha=1.0, beta=1.0, C=C[5])
        assert torch.equal(Y, (want + C[5].double()).float())


@pytest.mark.parametrize("transposed,x,n,k,s", [(False, "f32", 16385, 5500, 10100), (True, "f32", 16385, 5500, 10100), (False, "mx4", 16385, 16500, 10100)])
def test_more_tiles_of_long_sums_than_one_launch_takes(lib, torch, transposed, x, n, k, s):
    g = torch.Generator(device="cuda").manual_seed(16)
    q, r = (k, n) if transposed else (n, k)
    codes, scales, A = whole_codes(torch, q, r, g)
    M = lib.MXMatrix(codes, scales, r, lib.CODED_MX4)
    A = A.t() if transposed else A
    X, X64 = dense_whole(torch, x, s, k, True, g)
    if x == "mx4":
        X = lib.MXMatrix(*X, k, lib.CODED_MX4)
    Y = torch.empty((s, n), device="cuda")
    (lib.coded_mx_mm_t if transposed else lib.coded_mx_mm)(M, X, Y, x_rows=True, y_rows=True)
    S = X64 @ A.t()
    assert float(S.abs().max()) < 2 ** 24
    assert torch.equal(Y.double(), S)


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("x", ["f32", "bf16", "mx4"])
@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("s", [512, 2048])
def test_small_terms_beside_a_large_one_are_lost_to_one_chain_at_most(lib, torch, transposed, x, y, s):
    """Sums of 2^24, 31 zeros and k - 32 terms of 2^-6, by splits of tiles and by whole ones.  Next to 2^24 (fp32
    numbers there are 2 apart) the small terms may go missing, but those of the large term's chain alone, 16384 (bf16
    results: 65536): every other chain is exact, and adding up the chains' and splits' sums, at most 64 + k / 16384 of
    them, loses up to 2 each."""
    if transposed and x == "mx4":
        pytest.skip("U is dense")
    n, k = 8192, 262144
    q, r = (k, n) if transposed else (n, k)
    sign = torch.where(torch.arange(n, device="cuda") % 3 == 0, -1.0, 1.0)
    nibble = torch.where(sign < 0, 0xA, 0x2).to(torch.uint8)   # -1, 1
    if transposed:
        codes = (nibble[0::2] | nibble[1::2] << 4).repeat(q, 1)
    else:
        codes = (nibble | nibble << 4)[:, None].repeat(1, r // 2)
    M = lib.MXMatrix(codes, torch.full((q, r // 32), 127, dtype=torch.uint8, device="cuda"), r, lib.CODED_MX4)
    if x == "mx4":
        xc = torch.full((s, k // 2), 0x22, dtype=torch.uint8, device="cuda")
        xc[:, 1:16] = 0
        xc[:, 0] = 2
        xs = torch.full((s, k // 32), 127 - 6, dtype=torch.uint8, device="cuda")
        xs[:, 0] = 127 + 24
        X = lib.MXMatrix(xc, xs, k, lib.CODED_MX4)
    else:
        X = torch.full((s, k), 2.0 ** -6, dtype=torch.float32 if x == "f32" else torch.bfloat16, device="cuda")
        X[:, 1:32] = 0
        X[:, 0] = 2.0 ** 24
    C = (-2.0 ** 24 * sign).to(torch.bfloat16 if y == "bf16" else torch.float32)
    Y = torch.empty((s, n), dtype=C.dtype, device="cuda")
    (lib.coded_mx_mm_t if transposed else lib.coded_mx_mm)(M, X, Y, x_rows=True, y_rows=True, beta=1.0, C=C)
    want = (k - 32) * 2.0 ** -6
    bound = (65536 if y == "bf16" else 16384) * 2.0 ** -6 + 2 * (64 + k / 16384) + (2.0 ** -8 * want if y == "bf16" else 0)
    worst = float((Y.double() * sign - want).abs().max())
    assert worst <= bound, (worst, bound)


@pytest.mark.parametrize("transposed,x,s,x_rows,k", [(True, "bf16", 17, False, (1 << 22) + 37), (True, "bf16", 18, False, (1 << 22) + 37),
                                                     (True, "f32", 6, False, (1 << 22) + 37), (False, "bf16", 65, False, (1 << 22) + 37),
                                                     (False, "bf16", 65, True, (1 << 22) + 37), (False, "bf16", 65, True, (1 << 22) + 64),
                                                     (False, "bf16", 65, True, (1 << 23) + 64), (True, "bf16", 66, True, (1 << 23) + 64)])
def test_millions_of_terms(lib, torch, transposed, x, s, x_rows, k):
    """More terms, and rows of X further apart, than 32-bit offsets within a tile of such rows would take."""
    n = 40
    q, r = (k, n) if transposed else (n, k)
    g = torch.Generator(device="cuda").manual_seed(17)
    codes, scales, A = whole_codes(torch, q, r, g)
    keep = (torch.rand((q, codes.shape[1]), device="cuda", generator=g) < 0.03).to(torch.uint8)   # sums below 2^24
    codes *= keep
    A *= keep.repeat_interleave(2, 1)[:, :r]
    M = lib.MXMatrix(codes, scales, r, lib.CODED_MX4)
    A = A.t() if transposed else A
    X, X64 = dense_whole(torch, x, s, k, x_rows, g)
    Y = torch.empty((n, s), device="cuda")
    (lib.coded_mx_mm_t if transposed else lib.coded_mx_mm)(M, X, Y, x_rows=x_rows)
    want = A @ X64.t()
    assert float((A.abs() @ X64.t().abs()).max()) < 2 ** 24
    assert torch.equal(Y.double(), want)


@pytest.mark.parametrize("x", ["bf16", "mx8"])
def test_many_millions_of_right_hand_sides(lib, torch, x):
    """More of X than one launch copies or unpacks."""
    g = torch.Generator(device="cuda").manual_seed(18)
    n, k, s = 3, 63, ((1 << 26) if x == "bf16" else (1 << 25)) + 1000
    codes, scales, A = whole_codes(torch, n, k, g)
    M = lib.MXMatrix(codes, scales, k, lib.CODED_MX4)
    if x == "bf16":
        X = torch.empty((s, k), dtype=torch.bfloat16, device="cuda").random_(-7, 8, generator=g)
    else:
        xc = torch.empty((s, 64), dtype=torch.uint8, device="cuda").random_(0x38, 0x40, generator=g)   # 1 to 1.875
        xc[:, 63] = 0
        X = lib.MXMatrix(xc, torch.full((s, 4), 127, dtype=torch.uint8, device="cuda"), k, lib.CODED_MX8)
    Y = torch.empty((s, n), device="cuda")
    lib.coded_mx_mm(M, X, Y, x_rows=True, y_rows=True)
    for at in range(0, s, 1 << 22):
        rows = slice(at, min(s, at + (1 << 22)))
        v = X[rows].double() if x == "bf16" else torch.tensor(om.format_values(8), device="cuda")[xc[rows, :63].int()]
        assert torch.equal(Y[rows].double(), v @ A.t()), at
