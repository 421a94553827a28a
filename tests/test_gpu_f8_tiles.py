"""Products of 8-bit matrices whose sizes choose each kernel of them, against 64 bits on the device.

Bounds as in test_gpu_f8.py: (128 + blocks + 64) * 2^-23 of the sum of the terms' magnitudes; for bf16 results 7 * 2^-13 of
the largest of each eight consecutive terms where the 8-bit instruction is used, and half a step of the type, 2^-8.
"""
import pytest

from tests.gpu_helpers import torch_mod

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    t = torch_mod()
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    return t


def random_matrix(lib, torch, g, rows, cols, block_rows):
    """Any codes but NaN, and scales over sixteen powers of two: no two blocks could stand for each other."""
    blocks, groups = -(-cols // 128), -(-rows // block_rows)
    codes = torch.randint(0, 256, (rows, blocks * 128), generator=g, device="cuda", dtype=torch.uint8)
    codes[(codes & 0x7F) == 0x7F] = 0x7E
    codes[:, cols:] = 0
    scales = torch.rand((blocks, groups), generator=g, device="cuda") + 1
    scales = torch.ldexp(scales, torch.randint(-12, 4, (blocks, groups), generator=g, device="cuda"))
    return lib.F8Matrix(codes, scales, rows, cols, block_rows)


def values(torch, M):
    """What a matrix stands for, in 64 bits (whole blocks of columns)."""
    v = M.codes.view(torch.float8_e4m3fn).to(torch.float32).double()
    per = M.scales.t().double()
    per = per if M.block_rows == 1 else per.repeat_interleave(M.block_rows, 0)[:M.rows_]
    return (v.view(M.rows_, -1, 128) * per[:, :, None]).view(M.rows_, -1)


def largest_of_eights(torch, a, x):
    """For each result the largest of each eight consecutive terms' magnitudes, added up over the eights."""
    a, x = a.abs().float().t().contiguous(), x.abs().float().t().contiguous()
    total = torch.zeros((a.shape[1], x.shape[1]), device="cuda")
    most, one = torch.empty_like(total), torch.empty_like(total)
    for k in range(0, a.shape[0], 8):
        torch.mul(a[k, :, None], x[k, None, :], out=most)
        for i in range(k + 1, k + 8):
            torch.mul(a[i, :, None], x[i, None, :], out=one)
            torch.maximum(most, one, out=most)
        total += most
    return total.double() * (1 + 2.0 ** -10)


def check(lib, torch, q, r, s, y, block, x_block, cut, C=False, workspace=None):
    """Both orders of Y.  cut: the 8-bit instruction may be used, so bf16 results may be off by its cut."""
    g = torch.Generator(device="cuda").manual_seed(q * 7 + s * 3 + r + block)
    A, X = random_matrix(lib, torch, g, q, r, block), random_matrix(lib, torch, g, s, r, x_block)
    a, x = values(torch, A), values(torch, X)
    want, size = a @ x.t().contiguous(), a.abs() @ x.abs().t().contiguous()
    bound = (128 + -(-r // 128) + 64) * 2.0 ** -23 * size + 2.0 ** -22 * want.abs()
    if y == "bf16" and cut:
        bound += 7 * 2.0 ** -13 * largest_of_eights(torch, a, x)
    dt = torch.bfloat16 if y == "bf16" else torch.float32
    for y_rows in (False, True):
        w, b = (want.t(), bound.t()) if y_rows else (want, bound)
        c = torch.randn(w.shape, generator=g, device="cuda").to(dt) if C else None
        if C:
            w = w - 3.0 * c.double()
            b = b + 2.0 ** -22 * (w.abs() + 3.0 * c.double().abs())
        if y == "bf16":
            b = b + 2.0 ** -8 * (w.abs() + b)
        wide = torch.full((w.shape[0] + 2, w.shape[1] + 3), 7.0, dtype=dt, device="cuda")
        Y = wide[1:-1, :w.shape[1]]
        lib.coded_f8_mm(A, X, Y, y_rows=y_rows, beta=-3.0 if C else 0.0, C=c)
        off = ((Y.double() - w).abs() / b).max()
        assert bool(off <= 1), float(off)     # a NaN is not
        assert bool((wide[0] == 7).all()) and bool((wide[-1] == 7).all()) and bool((wide[:, w.shape[1]:] == 7).all())


BLOCKS = [(128, 1), (1, 1), (128, 128)]


@pytest.mark.parametrize("block,x_block", BLOCKS)
@pytest.mark.parametrize("y,q,r,s,shared", [
    ("f32", 4340, 4090, 2290, 306 - 256), ("bf16", 4340, 4090, 4350, 289 - 256), ("f32", 4090, 4090, 2040, 0), ("bf16", 4090, 4100, 4090, 0)])
def test_large_tiles(lib, torch, y, q, r, s, shared, block, x_block):
    """Tiles of 128 x 256 (fp32 results) and 256 x 256 (bf16): one whole round of 256, and `shared` more whose sums are split
    four ways, as the workspace shows; ends inside tiles and blocks."""
    tile = 128 * 256 if y == "f32" else 256 * 256
    for y_rows in (False, True):
        assert lib.coded_f8_workspace(q, r, s, lib.CODED_F32 if y == "f32" else lib.CODED_BF16, y_rows) == shared * 4 * tile * 4
    check(lib, torch, q, r, s, y, block, x_block, cut=True, C=shared > 0)


@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("block,x_block", BLOCKS)
@pytest.mark.parametrize("s", [1, 9, 17, 32])
def test_few_sides_32_results_a_workgroup(lib, torch, s, y, block, x_block):
    """From 16353 results on a workgroup takes 32 of them; the last one has 17."""
    check(lib, torch, 16401, 300, s, y, block, x_block, cut=False)


@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("block,x_block", BLOCKS)
@pytest.mark.parametrize("q,r,s", [(70001, 4096, 1), (70001, 4096, 16), (70001, 4096, 17), (7993, 40000, 5), (1000, 300000, 16)])
def test_few_sides_of_a_streamed_matrix(lib, torch, q, r, s, y, block, x_block):
    """More than 256 MB of codes, read with non-temporal loads: 32 and 16 results a workgroup, whole and split sums, and from
    17 right-hand sides on tiles."""
    check(lib, torch, q, r, s, y, block, x_block, cut=s > 16)


def test_few_sides_take_33_in_tiles(lib, torch):
    for s, cut in ((32, False), (33, True)):
        for y in ("f32", "bf16"):
            check(lib, torch, 5000, 1000, s, y, 128, 1, cut, C=True)


# ---------------------------------------------------------------- workspaces that the caller gives

def guarded(torch, n):
    """n bytes, 256-byte aligned, between bytes of 0xA5."""
    whole = torch.full((n + 512,), 0xA5, dtype=torch.uint8, device="cuda")
    return whole, whole[256:256 + n]


@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("q,r,s", [(16, 40000, 1), (300, 16384, 260), (260, 16384, 20), (4340, 4090, 4350)])
def test_products_stay_within_a_given_workspace(lib, torch, q, r, s, y):
    g = torch.Generator(device="cuda").manual_seed(r)
    A, X = random_matrix(lib, torch, g, q, r, 128), random_matrix(lib, torch, g, s, r, 1)
    dt = torch.bfloat16 if y == "bf16" else torch.float32
    n = lib.coded_f8_workspace(q, r, s, lib.CODED_BF16 if y == "bf16" else lib.CODED_F32, True)
    assert n > 0
    want = torch.empty(s, q, dtype=dt, device="cuda")
    lib.coded_f8_mm(A, X, want, y_rows=True)
    for _ in range(2):
        whole, ws = guarded(torch, n)
        got = torch.full((s, q), float("nan"), dtype=dt, device="cuda")
        lib.coded_f8_mm(A, X, got, y_rows=True, workspace=ws)
        assert torch.equal(got, want)
        assert bool((whole[:256] == 0xA5).all()) and bool((whole[256 + n:] == 0xA5).all())


@pytest.mark.parametrize("n,vocab,d", [(1, 3, 5), (1000, 40, 33), (4096, 70, 8), (4097, 300, 17), (70000, 5, 300)])
def test_gradients_stay_within_a_given_workspace(lib, torch, n, vocab, d):
    g = torch.Generator(device="cuda").manual_seed(n)
    tok = torch.randint(0, vocab, (n,), generator=g, device="cuda")
    G = torch.randn(n, d, generator=g, device="cuda")
    want = torch.empty(vocab, d, device="cuda")
    lib.coded_embed_grad(G, tok, want)
    size = lib.coded_embed_workspace(n, vocab, d)
    whole, ws = guarded(torch, size)
    got = torch.full((vocab, d), float("nan"), device="cuda")
    lib.coded_embed_grad(G, tok, got, workspace=ws)
    assert torch.equal(got, want)
    assert bool((whole[:256] == 0xA5).all()) and bool((whole[256 + size:] == 0xA5).all())


# ---------------------------------------------------------------- more rows than one launch takes

def test_a_transpose_stored_in_two_launches(lib, torch):
    """A column of 2^30 + 300 rows, one row of its transpose; a launch takes 2^23 tiles of 128 rows."""
    q = (1 << 30) + 300
    a = torch.zeros(q, 1, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 127, 128, (1 << 30) - 1, 1 << 30, (1 << 30) + 128, q - 1], device="cuda")
    a[at, 0] = torch.tensor([3.0, -1.0, 5.0, 7.0, -9.0, 11.0, 13.0], device="cuda").bfloat16()
    MT = lib.alloc_f8(1, q)
    MT.codes.fill_(0xFF)
    MT.scales.fill_(float("nan"))
    lib.coded_f8_quantize(a, None, MT)
    # each is its block's largest, but -1: 448 times the scale, which is a 448th of it
    want = torch.full((7,), 448.0, device="cuda") * torch.tensor([1, -1 / 3, 1, 1, -1, 1, 1], device="cuda")
    code = MT.codes[0, at].view(torch.float8_e4m3fn).float()
    assert bool(((code - want).abs() <= 2.0 ** -4 * want.abs()).all())
    assert torch.equal(MT.scales[at // 128, 0], torch.tensor([3.0, 3, 5, 7, 9, 11, 13], device="cuda") / torch.full((7,), 448.0, device="cuda"))
    assert int((MT.codes[0] != 0).sum()) == 7
    empty = torch.tensor([2.0 ** -100], device="cuda") / torch.tensor([448.0], device="cuda")
    assert int((MT.scales[:, 0] == empty).sum()) == MT.scales.shape[0] - 6


def test_reading_back_in_two_launches(lib, torch):
    """Rows of 2049 columns take two pieces: a launch takes 2^22 of them."""
    q, r = (1 << 22) + 130, 2049
    M = lib.alloc_f8(q, r, 128)
    M.codes.fill_(0x38)             # ones
    M.codes[:, 2048:] = 0x40        # and a two
    M.scales.copy_(torch.arange(M.scales.shape[1], device="cuda").expand(M.scales.shape))
    out = torch.full((q + 1, r), -1.0, dtype=torch.bfloat16, device="cuda")
    lib.coded_f8_dequantize(M, out[:q])
    rows = torch.arange(q, device="cuda") // 128
    for c, times in ((0, 1), (2047, 1), (2048, 2)):
        assert torch.equal(out[:q, c], (rows * times).float().bfloat16())
    assert bool((out[q] == -1).all())
    low, high = out[:q, :2048].min(1).values, out[:q, :2048].max(1).values
    assert torch.equal(low, high)


def test_dropout_in_two_launches(lib, torch):
    """2^22 rows of 2049 columns to a launch; the rows behind it are those of a batch of their own that begins there."""
    q, r = (1 << 22) + 70, 2049
    x = torch.ones(q, r, dtype=torch.bfloat16, device="cuda")
    lib.coded_dropout(x, x, 0.5, 11, 12)
    for at in (0, (1 << 22) - 64, (1 << 22) - 3, 1 << 22, q - 64):
        part = torch.ones(64, r, dtype=torch.bfloat16, device="cuda")
        lib.coded_dropout(part, part, 0.5, 11, 12, first_row=at)
        assert torch.equal(x[at:at + 64], part)


def test_lookup_in_two_launches(lib, torch):
    n, d = (1 << 22) + 50, 2049
    E = torch.randn(37, d, device="cuda").bfloat16()
    tok = (torch.arange(n, device="cuda") * 7919 % 37).int()
    out = torch.zeros(n + 1, d, dtype=torch.bfloat16, device="cuda")
    lib.coded_embed(E, tok, out[:n])
    for at in range(0, n, 1 << 18):
        end = min(n, at + (1 << 18))
        assert torch.equal(out[at:end], E[tok[at:end].long()])
    assert bool((out[n] == 0).all())
