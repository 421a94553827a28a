"""Matrices in 8 bits with blocks of 128 on the GPU against the oracle in 64 bits.

Bounds of a product.  A product of two codes is exact in fp32.  A block's 128 products are added in fp32, whatever
the order, within 128 * 2^-23 of the sum of their magnitudes; the product of two scales, and that with the sum,
round once each; with b blocks, b additions, and the few that join splits and waves, round once each.  So a result
is within (128 + b + 64) * 2^-23 of the sum of the terms' magnitudes ("size"), plus 2^-22 of the result and of beta C
for the epilogue.  For bf16 results the 8-bit matrix instruction cuts each of eight consecutive terms off at
2^-13 of the largest of them: up to 7 * 2^-13 of that, summed over the eights ("largest"); the rounding to bf16 is
half a step, 2^-8 of the value.  Whole numbers small enough are exact.
"""
import numpy as np
import pytest

from oracle import f8 as of
from oracle.mx import format_values
from tests.gpu_helpers import torch_mod

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    t = torch_mod()
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    return t


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


def dense(torch, a, dtype, pad=0):
    """a on the device, in rows `pad` elements further apart, NaN between them."""
    wide = np.full((a.shape[0], a.shape[1] + pad), np.nan, np.float32)
    wide[:, :a.shape[1]] = a
    return torch.from_numpy(wide).cuda().to(dtype)[:, :a.shape[1]]


def stored(lib, torch, rng, rows, cols, block_rows, pad=0, whole=False):
    """(F8Matrix, fp64 values).  whole: scales of 1 and whole codes.  pad: 16-byte pieces of 0x7F (NaN) behind each row
    of codes, NaN behind each row of scales."""
    blocks, groups = -(-cols // 128), -(-rows // block_rows)
    if whole:
        pick = [c for c, v in enumerate(format_values(8)) if np.isfinite(v) and v == round(v) and abs(v) <= 8]
        codes = np.array(pick, dtype=np.uint8)[rng.integers(0, len(pick), (rows, blocks * 128))]
        scales = np.ones((blocks, groups), dtype=np.float32)
    else:
        codes = rng.integers(0, 256, (rows, blocks * 128)).astype(np.uint8)
        codes[(codes & 0x7F) == 0x7F] = 0x7E
        scales = (rng.random((blocks, groups)) * 2.0 ** rng.integers(-12, 4, (blocks, groups)) + 2.0 ** -20).astype(np.float32)
    codes[:, cols:] = 0
    v = of.values(codes, scales, cols, block_rows)
    c = np.concatenate([codes, np.full((rows, 16 * pad), 0x7F, np.uint8)], 1)
    s = np.concatenate([scales, np.full((blocks, pad), np.nan, np.float32)], 1)
    return lib.F8Matrix(torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda(), rows, cols, block_rows), v


def limits(a, x):
    """(product, size, largest) of two matrices' rows."""
    pad = -a.shape[1] % 8
    ma, mx = np.pad(np.abs(a), ((0, 0), (0, pad))), np.pad(np.abs(x), ((0, 0), (0, pad)))
    largest = np.zeros((a.shape[0], x.shape[0]))
    for k in range(0, ma.shape[1], 8):
        largest += (ma[:, None, k:k + 8] * mx[None, :, k:k + 8]).max(2)
    return a @ x.T, ma @ mx.T, largest


def check_product(lib, torch, rng, q, r, s, y, y_rows, block=128, x_block=1, pad=0, alpha=1.0, beta=0.0, whole=False, bias=False):
    A, av = stored(lib, torch, rng, q, r, block, pad, whole)
    X, xv = stored(lib, torch, rng, s, r, x_block, pad, whole)
    dt = torch.bfloat16 if y == "bf16" else torch.float32
    shape = (s, q) if y_rows else (q, s)
    wide = torch.full((shape[0] + 2, shape[1] + pad), 7.0, dtype=dt, device="cuda")
    Y = wide[1:-1, :shape[1]]
    cv, C = 0.0, None
    if beta:
        cv = torch.from_numpy(rng.standard_normal((1, shape[1]) if bias else shape).astype(np.float32)).to(dt).float().numpy().astype(np.float64)
        C = dense(torch, cv, dt, pad)[0] if bias else dense(torch, cv, dt, pad)
    if whole:      # exact in 64 bits wherever it is computed
        want = (torch.from_numpy(av).cuda() @ torch.from_numpy(np.ascontiguousarray(xv.T)).cuda()).cpu().numpy()
    else:
        want, size, largest = limits(av, xv)
        if y_rows:
            size, largest = size.T, largest.T
    want = alpha * (want.T if y_rows else want) + beta * cv
    lib.coded_f8_mm(A, X, Y, y_rows=y_rows, alpha=alpha, beta=beta, C=C)
    torch.cuda.synchronize()
    got = host(Y)
    if whole:
        assert np.array_equal(got, want if y == "f32" else host(torch.from_numpy(want).to(dt)))
    else:
        bound = abs(alpha) * (128 + -(-r // 128) + 64) * 2.0 ** -23 * size + 2.0 ** -22 * (np.abs(want) + np.abs(beta * cv)) + 2.0 ** -120
        if y == "bf16":
            bound = bound + abs(alpha) * 7 * 2.0 ** -13 * largest
            bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
        assert np.all(np.abs(got - want) <= bound), np.max(np.abs(got - want) / bound)
    # nothing around the result is touched
    assert bool((wide[0] == 7).all()) and bool((wide[-1] == 7).all()) and bool((wide[:, shape[1]:] == 7).all())


# ---------------------------------------------------------------- storing

def codes_of(M):
    """Codes (whole blocks) and scales on the host."""
    n, g = -(-M.cols // 128), -(-M.rows_ // M.block_rows)
    return M.codes.cpu().numpy()[:, :n * 128], M.scales.cpu().numpy()[:n, :g]


def room(lib, torch, q, r, block, pad):
    n, g = -(-r // 128), -(-q // block)
    codes = torch.full((q + 1, n * 128 + 16 * pad), 0xAB, dtype=torch.uint8, device="cuda")
    scales = torch.full((n + 1, g + pad), 7.0, dtype=torch.float32, device="cuda")
    return lib.F8Matrix(codes[:q], scales, q, r, block), codes, scales, n, g


@pytest.mark.parametrize("block,t_block", [(1, 1), (128, 128), (1, 128), (128, 1), (1, None), (None, 1), (128, None), (None, 128)])
@pytest.mark.parametrize("q,r,dtype,pad", [(1, 1, "f32", 0), (1, 129, "bf16", 1), (7, 128, "f32", 3), (128, 127, "bf16", 0), (129, 8, "f32", 1),
                                           (130, 260, "bf16", 5), (257, 131, "f32", 0)])
def test_stored_codes_equal_the_oracles(lib, torch, q, r, dtype, pad, block, t_block):
    rng = np.random.default_rng(q * 10007 + r * 11)
    a = (rng.standard_normal((q, r)) * 2.0 ** rng.integers(-10, 10, (q, r))).astype(np.float32)
    a[rng.random((q, r)) < 0.3] *= 0
    a[rng.random(q) < 0.1] = 0
    near = rng.random((q, r)) < 0.3        # ties and edges where a block's largest value is 448 2^k
    a[near] = rng.choice([448, 17, 19, 23.5, 2.0 ** -10, 3 * 2.0 ** -10, -0.0, -464, 432, 1e-38, 1e-45], near.sum())
    A = dense(torch, a, torch.bfloat16 if dtype == "bf16" else torch.float32, pad)
    M = MT = None
    if block:
        M, codes, scales, n, g = room(lib, torch, q, r, block, pad)
    if t_block:
        MT, t_codes, t_scales, tn, tg = room(lib, torch, r, q, t_block, pad)
    lib.coded_f8_quantize(A, M, MT)
    torch.cuda.synchronize()
    for m, v, b in ((M, host(A), block), (MT, host(A).T, t_block)):
        if m is None:
            continue
        want_c, want_s = of.quantize(v, b)
        got_c, got_s = codes_of(m)
        assert np.array_equal(got_s, want_s) and np.array_equal(got_c, want_c)
        for dt in (torch.float32, torch.bfloat16):
            out = torch.full((m.rows_, m.cols + pad), 7.0, dtype=dt, device="cuda")
            lib.coded_f8_dequantize(m, out[:, :m.cols])
            back = torch.from_numpy(of.values(want_c, want_s, m.cols, b).astype(np.float32)).to(dt)   # one rounding of an exact product
            assert np.array_equal(host(out[:, :m.cols]), host(back))
            assert bool((out[:, m.cols:] == 7).all())
    for wide, rows, cols in ((codes, q, n * 128), (scales, n, g)) if block else ():
        edge = 0xAB if wide.dtype == torch.uint8 else 7.0
        assert bool((wide[rows:] == edge).all()) and bool((wide[:, cols:] == edge).all())
    for wide, rows, cols in ((t_codes, r, tn * 128), (t_scales, tn, tg)) if t_block else ():
        edge = 0xAB if wide.dtype == torch.uint8 else 7.0
        assert bool((wide[rows:] == edge).all()) and bool((wide[:, cols:] == edge).all())


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_blocks_without_values_hide_nothing(lib, torch, bad):
    a = torch.ones(260, 300, device="cuda")
    a[130, 5] = bad
    M, MT = lib.alloc_f8(260, 300), lib.alloc_f8(300, 260)
    W = lib.alloc_f8(260, 300, 128)
    lib.coded_f8_quantize(a, M, MT)
    lib.coded_f8_quantize(a, W)
    for m, where in ((M, np.s_[130:131, 0:128]), (MT, np.s_[5:6, 128:256]), (W, np.s_[128:256, 0:128])):
        out = torch.empty(m.shape, device="cuda")
        lib.coded_f8_dequantize(m, out)
        nan = np.zeros(m.shape, dtype=bool)
        nan[where] = True
        got = host(out)
        assert np.array_equal(np.isnan(got), nan) and np.all(np.abs(got[~nan] - 1) <= 2.0 ** -22)
        assert bool((m.codes[:, :m.cols][torch.from_numpy(nan).cuda()] == 0).all())


def test_nothing_to_store(lib, torch):
    for q, r in ((0, 5), (5, 0), (0, 0)):
        lib.coded_f8_quantize(torch.empty(q, r, device="cuda"), lib.alloc_f8(q, r), lib.alloc_f8(r, q))
        lib.coded_f8_dequantize(lib.alloc_f8(q, r), torch.empty(q, r, device="cuda"))


def test_runs_of_rows_are_matrices(lib, torch):
    rng = np.random.default_rng(5)
    for block in (1, 128):
        W, wv = stored(lib, torch, rng, 300, 200, block)
        X, xv = stored(lib, torch, rng, 9, 200, 1)
        part = W.rows(128, 290)
        Y = torch.empty(162, 9, device="cuda")
        lib.coded_f8_mm(part, X, Y)
        want, size, _ = limits(wv[128:290], xv)
        assert np.all(np.abs(host(Y) - want) <= 200 * 2.0 ** -23 * size)


# ---------------------------------------------------------------- products

SIZES = [(1, 1, 1), (3, 127, 2), (16, 128, 16), (17, 129, 1), (65, 300, 33), (130, 1000, 5), (5, 640, 130), (200, 256, 70), (129, 513, 129), (300, 130, 300)]


@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("y_rows", [False, True])
@pytest.mark.parametrize("q,r,s", SIZES)
def test_product(lib, torch, q, r, s, y, y_rows):
    check_product(lib, torch, np.random.default_rng(q + 1000 * s + r), q, r, s, y, y_rows)


@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("block,x_block", [(1, 1), (1, 128), (128, 128)])
@pytest.mark.parametrize("q,r,s", [(130, 257, 3), (150, 390, 140), (257, 128, 129)])
def test_product_of_any_blocks(lib, torch, q, r, s, block, x_block, y):
    for y_rows in (False, True):
        check_product(lib, torch, np.random.default_rng(q + s), q, r, s, y, y_rows, block, x_block)


@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("q,r,s", [(33, 200, 4), (140, 300, 150)])
def test_alpha_beta_bias_and_strides(lib, torch, q, r, s, y):
    rng = np.random.default_rng(q)
    for y_rows in (False, True):
        for alpha, beta, bias in ((-0.5, 1.0, False), (2.0, -3.0, True), (0.0, 1.0, False)):
            check_product(lib, torch, rng, q, r, s, y, y_rows, pad=3, alpha=alpha, beta=beta, bias=bias)


@pytest.mark.parametrize("q,r,s,y", [(16, 40000, 1, "f32"), (40, 20000, 20, "bf16"), (300, 16384, 260, "f32"), (300, 16384, 260, "bf16"), (600, 2000, 700, "f32"),
                                     (600, 2000, 700, "bf16"), (4100, 300, 2100, "bf16"), (2100, 640, 1030, "f32"), (70, 50000, 90, "bf16")])
@pytest.mark.parametrize("block,x_block", [(128, 1), (1, 1)])
def test_whole_numbers_are_exact(lib, torch, q, r, s, y, block, x_block):
    """Many tiles, and sums split among workgroups: whole numbers below 2^24, exact in whatever order."""
    rng = np.random.default_rng(r)
    for y_rows in (False, True):
        check_product(lib, torch, rng, q, r, s, y, y_rows, block, x_block, whole=True)


def test_result_may_be_c(lib, torch):
    rng = np.random.default_rng(1)
    for q, s in ((40, 3), (300, 280)):
        A, av = stored(lib, torch, rng, q, 256, 128)
        X, xv = stored(lib, torch, rng, s, 256, 1)
        c = rng.standard_normal((s, q)).astype(np.float32)
        Y = torch.from_numpy(c).cuda()
        lib.coded_f8_mm(A, X, Y, y_rows=True, beta=1.0, C=Y)
        want, size, _ = limits(xv, av)
        assert np.all(np.abs(host(Y) - want - c) <= 200 * 2.0 ** -23 * size + 2.0 ** -22 * (np.abs(c) + np.abs(want)))


def test_sum_of_no_terms(lib, torch):
    A, X = lib.alloc_f8(5, 0, 128), lib.alloc_f8(3, 0)
    Y, C = torch.full((3, 5), 9.0, device="cuda"), torch.arange(15.0, device="cuda").view(3, 5)
    lib.coded_f8_mm(A, X, Y, y_rows=True)
    assert bool((Y == 0).all())
    lib.coded_f8_mm(A, X, Y, y_rows=True, beta=2.0, C=C)
    assert torch.equal(Y, 2 * C)


@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("q,s", [(40, 3), (300, 280)])
def test_nan_reaches_its_own_results_alone(lib, torch, q, s, y):
    rng = np.random.default_rng(2)
    A, av = stored(lib, torch, rng, q, 300, 1)
    X, xv = stored(lib, torch, rng, s, 300, 1)
    A.codes[q - 2, 130] = 0x7F      # a code that is no number
    X.scales[1, s - 1] = float("nan")   # a block without values
    X.codes[s - 1, 128:256] = 0
    Y = torch.empty(q, s, dtype=torch.bfloat16 if y == "bf16" else torch.float32, device="cuda")
    lib.coded_f8_mm(A, X, Y)
    want = np.zeros((q, s), dtype=bool)
    want[q - 2] = True
    want[:, s - 1] = True
    assert np.array_equal(np.isnan(host(Y)), want) and np.all(np.isfinite(host(Y)[~want]))


def test_no_results(lib, torch):
    lib.coded_f8_mm(lib.alloc_f8(0, 5), lib.alloc_f8(3, 5), torch.empty(0, 3, device="cuda"))
    lib.coded_f8_mm(lib.alloc_f8(5, 5), lib.alloc_f8(0, 5), torch.empty(5, 0, device="cuda"))


def test_on_another_stream_and_twice(lib, torch):
    """Calls on two streams at once, each with a workspace of its own stream, give what they give alone."""
    rng = np.random.default_rng(3)
    A, _ = stored(lib, torch, rng, 32, 30000, 128)
    X, _ = stored(lib, torch, rng, 2, 30000, 1)
    B, _ = stored(lib, torch, rng, 300, 8192, 128)
    Z, _ = stored(lib, torch, rng, 280, 8192, 1)
    want, want2 = torch.empty(32, 2, device="cuda"), torch.empty(300, 280, device="cuda")
    lib.coded_f8_mm(A, X, want)
    lib.coded_f8_mm(B, Z, want2)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for _ in range(10):
        got, got2 = torch.empty_like(want), torch.empty_like(want2)
        torch.cuda.synchronize()
        lib.coded_f8_mm(A, X, got, stream=streams[0])
        lib.coded_f8_mm(B, Z, got2, stream=streams[1])
        outs.append((got, got2))
    torch.cuda.synchronize()
    for got, got2 in outs:
        assert torch.equal(got, want) and torch.equal(got2, want2)


@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("q,s", [(40, 70), (300, 3)])
def test_sums_longer_than_one_chain(lib, torch, q, s, y):
    """600000 terms, 4688 blocks; whole numbers of at most 4 whose sums stay below 2^24."""
    rng = np.random.default_rng(q)
    r = 600000
    pick = np.array([c for c, v in enumerate(format_values(8)) if np.isfinite(v) and v == round(v) and abs(v) <= 4], dtype=np.uint8)

    def side(rows):
        codes = pick[rng.integers(0, len(pick), (rows, -(-r // 128) * 128))]
        codes[:, r:] = 0
        v = torch.from_numpy(format_values(8)[codes].astype(np.float32)).cuda()[:, :r]
        return lib.F8Matrix(torch.from_numpy(codes).cuda(), torch.ones(-(-r // 128), rows, device="cuda"), rows, r, 1), v

    A, av = side(q)
    X, xv = side(s)
    Y = torch.empty(s, q, dtype=torch.bfloat16 if y == "bf16" else torch.float32, device="cuda")
    lib.coded_f8_mm(A, X, Y, y_rows=True)
    want = (xv.double() @ av.double().t()).to(Y.dtype)
    assert torch.equal(Y, want)


def test_many_results_of_sums_longer_than_one_chain(lib, torch):
    """Ones times ones over 2^22 terms, scales 1 and 1 + 2^-12: a block's sum is 128 + 2^-5.  At most 4096 blocks to a
    workgroup, 1024 to a wave, then four waves and eight workgroups: within (1024 + 4 + 8 + 2) 2^-24 of the sum.  With all
    32768 blocks in one workgroup each wave's upper 4096 additions would lose half a step: 2^-13."""
    q, r = 4100, 1 << 22
    A = lib.F8Matrix(torch.full((q, r), 0x38, dtype=torch.uint8, device="cuda"), torch.ones(r // 128, -(-q // 128), device="cuda"), q, r, 128)
    X = lib.F8Matrix(torch.full((1, r), 0x38, dtype=torch.uint8, device="cuda"), torch.full((r // 128, 1), 1 + 2.0 ** -12, device="cuda"), 1, r, 1)
    Y = torch.zeros(q, device="cuda")
    lib.coded_f8_mm(A, X, Y)
    want = r * (1 + 2.0 ** -12)
    assert np.all(np.abs(host(Y) - want) <= (1024 + 4 + 8 + 2) * 2.0 ** -24 * want)


@pytest.mark.parametrize("y", ["f32", "bf16"])
def test_tiles_of_no_terms(lib, torch, y):
    dt = torch.bfloat16 if y == "bf16" else torch.float32
    A, X = lib.alloc_f8(300, 0, 128), lib.alloc_f8(280, 0)
    Y, C = torch.full((280, 300), 9.0, dtype=dt, device="cuda"), torch.randn(300, device="cuda").to(dt)
    lib.coded_f8_mm(A, X, Y, y_rows=True, beta=1.0, C=C)
    assert torch.equal(Y, C.expand(280, 300))


def test_a_matrix_times_itself(lib, torch):
    rng = np.random.default_rng(8)
    for rows in (20, 300):
        A, av = stored(lib, torch, rng, rows, 390, 1)
        Y = torch.empty(rows, rows, device="cuda")
        lib.coded_f8_mm(A, A, Y)
        want, size, _ = limits(av, av)
        # not symmetric to the bit: a sum t meets two scales one after the other, and fl(fl(t a) b) is not fl(fl(t b) a)
        assert np.all(np.abs(host(Y) - want) <= 200 * 2.0 ** -23 * size)


@pytest.mark.parametrize("q,r,s", [(65, 300, 33), (300, 640, 300)])
def test_two_results_at_once_share_nothing(lib, torch, q, r, s):
    """A workspace given by the caller; the same product twice into two results, and rows behind the last left as they were."""
    rng = np.random.default_rng(9)
    A, _ = stored(lib, torch, rng, q, r, 128)
    X, _ = stored(lib, torch, rng, s, r, 1)
    n = max(16, lib.coded_f8_workspace(q, r, s, lib.CODED_F32, False))
    outs = [torch.full((q + 3, s), 5.0, device="cuda") for _ in range(2)]
    for out in outs:
        lib.coded_f8_mm(A, X, out[:q], workspace=torch.empty(n, dtype=torch.uint8, device="cuda"))
    assert torch.equal(outs[0], outs[1]) and bool((outs[0][q:] == 5).all())


def test_many_short_rows_are_read_back(lib, torch):
    """More rows than one launch's workgroups take where rows lie side by side in them, and rows cut into pieces."""
    for q, r in ((1 << 20, 3), (3, 70000)):
        a = torch.randn(q, r, device="cuda")
        for block in (1, 128):
            M = lib.alloc_f8(q, r, block)
            lib.coded_f8_quantize(a, M)
            out = torch.empty(q, r, device="cuda")
            lib.coded_f8_dequantize(M, out)
            s = M.scales.t().repeat_interleave(block, 0)[:q].repeat_interleave(128, 1)[:, :r]
            assert bool(((out - a).abs() <= (2.0 ** -4 + 2.0 ** -20) * a.abs() + s * 2.0 ** -10).all())
