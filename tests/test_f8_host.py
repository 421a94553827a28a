"""Matrices in 8 bits, dropout and embeddings, what needs no GPU: the oracle's format and generator, the pitches,
and every refusal (all of them are found on the host before anything is launched)."""
import ctypes
import json
import math
import os

import numpy as np
import pytest

from oracle import f8 as of


def test_oracle_scale_and_codes():
    row = np.zeros((1, 130))
    row[0, :4] = [448, -224, 17, 2.0 ** -10]
    row[0, 128:] = [1, -1]
    c, s = of.quantize(row, 1)
    assert s.shape == (2, 1) and s[0, 0] == 1 and s[1, 0] == np.float32(1 / 448)
    assert list(of.values(c, s, 130, 1)[0, :4]) == [448, -224, 16, 0]     # 17 is between 16 and 18; a tie goes to the even code
    assert np.all(c[0, 130:] == 0)
    c, s = of.quantize(np.array([[1.0, math.inf], [0.0, 0.0]]), 1)
    assert math.isnan(s[0, 0]) and not c[0].any() and s[0, 1] == np.float32(2.0 ** -100 / 448)
    c, s = of.quantize(np.full((129, 1), 3.0), 128)
    assert s.shape == (1, 2) and np.all(c[:, 0] == 0x7E)


def test_oracle_quotients_are_single_roundings():
    """A stored maximum reads back as itself within two roundings, and never past the largest code."""
    rng = np.random.default_rng(0)
    v = rng.standard_normal((64, 128)).astype(np.float32)
    c, s = of.quantize(v, 1)
    back = of.values(c, s, 128, 1)
    at = np.argmax(np.abs(v), axis=1)
    top = v[np.arange(64), at].astype(np.float64)
    assert np.all(np.abs(back[np.arange(64), at] - top) <= 2.0 ** -24 * np.abs(top))
    # half a step of a code, and the roundings of scale, factor and product
    assert np.all(np.abs(back - v) <= (2.0 ** -4 + 2.0 ** -22) * np.abs(v) + s.T * 2.0 ** -10)


def test_oracle_words_are_the_published_generators():
    with open(os.path.join(os.path.dirname(__file__), "golden", "splitmix64_seed1234567.json")) as f:
        golden = json.load(f)
    outs = next(v for v in golden.values() if isinstance(v, list))
    assert [of.word(1234567, i) for i in range(len(outs))] == [int(v) for v in outs]


def test_oracle_mask_depends_on_place_alone():
    whole = of.kept(20, 7, 0.4, 5, 3, 100)
    assert np.array_equal(whole[6:11], of.kept(5, 7, 0.4, 5, 3, 106))
    assert 0.4 < whole.mean() < 0.8
    assert not np.array_equal(whole, of.kept(20, 7, 0.4, 5, 4, 100))


def test_oracle_skip_that_is_no_row_skips_none():
    E = np.array([[1.0], [2.0]])
    assert list(of.embed(E, np.array([0, 1]), 3.0, 0)[:, 0]) == [0, 6]
    for skip in (-1, 2):
        assert np.array_equal(np.isnan(of.embed(E, np.array([0, -1, 2]), 3.0, skip)[:, 0]), [False, True, True])


@pytest.mark.parametrize("q,r,block,want", [(0, 0, 1, (0, 0)), (1, 1, 1, (128, 1)), (300, 128, 128, (128, 3)), (129, 5750, 128, (5760, 2)), (7, 129, 1, (256, 7))])
def test_sizes(lib, q, r, block, want):
    assert lib.coded_f8_sizes(q, r, block) == want


def test_sizes_refused(lib):
    for args, status in [((1, 1, 2), "ARG"), ((-1, 1, 1), "SHAPE"), ((1, 2 ** 41, 1), "SHAPE")]:
        with pytest.raises(lib.CodedError) as e:
            lib.coded_f8_sizes(*args)
        assert e.value.status == getattr(lib, "CODED_ERR_" + status)


# A 6 x 200 matrix (pitches 256 and 6) with two right-hand sides: addresses that the checks look at and nothing reads.
MM = dict(q=6, r=200, s=2, br=1, codes=0x1000, ldc=256, scales=0x2000, lds=6, xbr=1, xc=0x3000, ldxc=256, xs=0x4000, ldxs=2, order=0,
          alpha=1.0, beta=0.0, C=None, ldcc=0, Y=0x5000, y_dt=0, ldy=2, ws=None, wsb=0, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(br=2), "ARG"), (dict(xbr=0), "ARG"), (dict(codes=None), "ARG"), (dict(scales=None), "ARG"), (dict(xc=None), "ARG"),
    (dict(xs=None), "ARG"), (dict(codes=0x1008), "ARG"), (dict(xc=0x3004), "ARG"), (dict(scales=0x2002), "ARG"), (dict(xs=0x4001), "ARG"),
    (dict(ldc=200), "SHAPE"), (dict(ldc=264), "SHAPE"), (dict(ldc=-256), "SHAPE"), (dict(ldxc=128), "SHAPE"), (dict(lds=5), "SHAPE"),
    (dict(ldxs=1), "SHAPE"), (dict(q=-1), "SHAPE"), (dict(r=-1), "SHAPE"), (dict(s=-1), "SHAPE"), (dict(q=2 ** 41, lds=2 ** 41), "SHAPE"),
    (dict(order=1), "ARG"), (dict(order=4), "ARG"), (dict(order=2), "SHAPE"), (dict(Y=None), "ARG"), (dict(Y=0x5002), "ARG"),
    (dict(y_dt=2), "ARG"), (dict(y_dt=4), "ARG"), (dict(ldy=1), "SHAPE"), (dict(alpha=math.inf), "ARG"), (dict(alpha=1e39), "ARG"),
    (dict(beta=math.nan), "ARG"), (dict(beta=1.0), "ARG"), (dict(beta=1.0, C=0x6000, ldcc=1), "SHAPE"),
    (dict(beta=1.0, C=0x6001, ldcc=2), "ARG"), (dict(beta=1.0, C=0x5000, ldcc=0), "ARG"),
    (dict(r=2 ** 23 + 1, ldc=2 ** 23 + 128, ldxc=2 ** 23 + 128), "UNSUPPORTED"), (dict(ldc=2 ** 24 + 16), "UNSUPPORTED"),
])
def test_product_refused(lib, change, status):
    assert lib.lib().coded_f8_mm(*{**MM, **change}.values()) == getattr(lib, "CODED_ERR_" + status)
    assert lib.last_error()


def test_product_without_results_is_fine_without_a_gpu(lib):
    assert lib.lib().coded_f8_mm(*{**MM, "s": 0}.values()) == lib.CODED_OK
    assert lib.lib().coded_f8_mm(*{**MM, "q": 0}.values()) == lib.CODED_OK


def test_product_needs_its_workspace(lib):
    # one right-hand side and few rows over a long sum: parts of it are added up in the workspace
    need = lib.coded_f8_workspace(16, 1 << 16, 1, lib.CODED_F32)
    assert need > 0
    a = {**MM, "q": 16, "r": 1 << 16, "s": 1, "ldc": 1 << 16, "ldxc": 1 << 16, "lds": 16}
    assert lib.lib().coded_f8_mm(*a.values()) == lib.CODED_ERR_ARG
    assert lib.lib().coded_f8_mm(*{**a, "ws": 0x7000, "wsb": need - 1}.values()) == lib.CODED_ERR_ARG
    assert lib.lib().coded_f8_mm(*{**a, "ws": 0x7008, "wsb": need}.values()) == lib.CODED_ERR_ARG


@pytest.mark.parametrize("q,r,s", [(4100, 1 << 22, 1), (20000, 1 << 23, 16), (7, 1 << 22, 20000), (100000, (1 << 19) + 1, 1), (2000, 1 << 23, 1)])
def test_few_right_hand_sides_have_bounded_chains(lib, q, r, s):
    """One workgroup adds at most 4096 blocks: longer sums leave their parts in the workspace, however many results there are."""
    for y in (lib.CODED_F32, lib.CODED_BF16):
        for y_rows in (False, True):
            parts = -(-r // 128 // 4096)
            assert lib.coded_f8_workspace(q, r, s, y, y_rows) >= parts * q * s * 4


def test_workspace_refused(lib):
    b = ctypes.c_int64()
    h = lib.lib()
    assert h.coded_f8_workspace(1, 1, 1, 0, 0, None) == lib.CODED_ERR_ARG
    for args, status in [((-1, 1, 1, 0, 0), "SHAPE"), ((1, 1, 2 ** 41, 0, 0), "SHAPE"), ((1, 2 ** 23 + 1, 1, 0, 0), "UNSUPPORTED"),
                         ((1, 1, 1, 3, 0), "ARG"), ((1, 1, 1, 0, 1), "ARG")]:
        assert h.coded_f8_workspace(*args, ctypes.addressof(b)) == getattr(lib, "CODED_ERR_" + status), args
    for args, status in [((-1, 1, 1), "SHAPE"), ((2 ** 31, 1, 1), "SHAPE"), ((1, 2 ** 31 - 1, 1), "SHAPE"), ((1, 1, -1), "SHAPE")]:
        assert h.coded_embed_workspace(*args, ctypes.addressof(b)) == getattr(lib, "CODED_ERR_" + status), args
    assert h.coded_embed_workspace(1, 1, 1, None) == lib.CODED_ERR_ARG


STORE = dict(dt=0, A=0x1000, q=3, r=200, lda=200, br=1, codes=0x2000, ldc=256, scales=0x3000, lds=3, tbr=1, tc=0x4000, ldtc=128, ts=0x5000,
             ldts=200, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(dt=2), "ARG"), (dict(dt=4), "ARG"), (dict(A=None), "ARG"), (dict(A=0x1002), "ARG"), (dict(lda=199), "SHAPE"), (dict(br=3), "ARG"),
    (dict(tbr=64), "ARG"), (dict(codes=None), "ARG"), (dict(scales=None), "ARG"), (dict(tc=None), "ARG"), (dict(ts=None), "ARG"),
    (dict(codes=0x2004), "ARG"), (dict(tc=0x4008), "ARG"), (dict(ldc=208), "SHAPE"), (dict(ldtc=112), "SHAPE"), (dict(lds=2), "SHAPE"),
    (dict(ldts=199), "SHAPE"), (dict(q=-1), "SHAPE"), (dict(r=-1), "SHAPE"),
    (dict(codes=None, scales=None, tc=None, ts=None), "ARG")])
def test_storing_refused(lib, change, status):
    assert lib.lib().coded_f8_quantize(*{**STORE, **change}.values()) == getattr(lib, "CODED_ERR_" + status)
    assert lib.last_error()


def test_reading_back_refused(lib):
    good = dict(q=3, r=200, br=1, codes=0x2000, ldc=256, scales=0x3000, lds=3, dt=0, out=0x1000, ldo=200, stream=None)
    for change, status in [(dict(br=2), "ARG"), (dict(codes=None), "ARG"), (dict(ldc=200), "SHAPE"), (dict(lds=2), "SHAPE"), (dict(dt=2), "ARG"),
                           (dict(out=None), "ARG"), (dict(out=0x1001), "ARG"), (dict(ldo=199), "SHAPE"), (dict(q=-1), "SHAPE")]:
        assert lib.lib().coded_f8_dequantize(*{**good, **change}.values()) == getattr(lib, "CODED_ERR_" + status), change


DROP = dict(dt=0, X=0x1000, q=3, r=5, ldx=5, p=0.5, seed=1, draw=2, first=0, C=None, ldcc=0, out=0x2000, ldo=5, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(dt=2), "ARG"), (dict(X=None), "ARG"), (dict(out=None), "ARG"), (dict(X=0x1002), "ARG"), (dict(ldx=4), "SHAPE"), (dict(ldo=4), "SHAPE"),
    (dict(C=0x3000, ldcc=4), "SHAPE"), (dict(C=0x3001, ldcc=5), "ARG"), (dict(p=-0.1), "ARG"), (dict(p=1.5), "ARG"), (dict(p=math.nan), "ARG"),
    (dict(draw=1 << 56), "ARG"), (dict(first=-1), "ARG"), (dict(first=(1 << 40) + 1), "ARG"), (dict(q=-1), "SHAPE"), (dict(r=2 ** 41, ldx=2 ** 41, ldo=2 ** 41), "SHAPE"),
    (dict(out=0x1000, ldo=6), "SHAPE"), (dict(C=0x2000, ldcc=7), "SHAPE")])
def test_dropout_refused(lib, change, status):
    assert lib.lib().coded_dropout(*{**DROP, **change}.values()) == getattr(lib, "CODED_ERR_" + status)


EMB = dict(e_dt=0, E=0x1000, vocab=10, d=5, lde=5, tok=0x2000, size=4, n=3, skip=-1, scale=1.0, o_dt=0, out=0x3000, ldo=5, stream=None)
GRAD = dict(g_dt=0, G=0x1000, n=3, d=5, ldg=5, tok=0x2000, size=4, vocab=10, skip=-1, scale=1.0, beta=0.0, e_dt=0, dE=0x3000, ldde=5, ws=None, wsb=0, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(e_dt=2), "ARG"), (dict(E=None), "ARG"), (dict(E=0x1001), "ARG"), (dict(lde=4), "SHAPE"), (dict(tok=None), "ARG"), (dict(tok=0x2002), "ARG"),
    (dict(size=2), "ARG"), (dict(size=8, tok=0x2004), "ARG"), (dict(n=-1), "SHAPE"), (dict(n=2 ** 31), "SHAPE"), (dict(vocab=-1), "SHAPE"),
    (dict(vocab=2 ** 31 - 1), "SHAPE"), (dict(d=-1), "SHAPE"), (dict(scale=math.inf), "ARG"), (dict(o_dt=3), "ARG"), (dict(out=None), "ARG"), (dict(ldo=4), "SHAPE")])
def test_lookup_refused(lib, change, status):
    assert lib.lib().coded_embed(*{**EMB, **change}.values()) == getattr(lib, "CODED_ERR_" + status)


@pytest.mark.parametrize("change,status", [
    (dict(g_dt=2), "ARG"), (dict(G=None), "ARG"), (dict(ldg=4), "SHAPE"), (dict(tok=None), "ARG"), (dict(size=1), "ARG"), (dict(n=-1), "SHAPE"),
    (dict(vocab=2 ** 31 - 1), "SHAPE"), (dict(scale=math.nan), "ARG"), (dict(beta=math.inf), "ARG"), (dict(e_dt=4), "ARG"), (dict(dE=None), "ARG"),
    (dict(ldde=4), "SHAPE"), (dict(), "ARG"), (dict(ws=0x4000, wsb=100), "ARG"), (dict(ws=0x4008, wsb=1 << 30), "ARG")])
def test_gradient_refused(lib, change, status):
    assert lib.lib().coded_embed_grad(*{**GRAD, **change}.values()) == getattr(lib, "CODED_ERR_" + status)


def test_wider_than_the_launches_reach(lib):
    w = 2 ** 27 + 1
    wide = {**STORE, "r": w, "lda": w, "ldc": 2 ** 27 + 128, "ldts": w}
    assert lib.lib().coded_f8_quantize(*wide.values()) == lib.CODED_ERR_UNSUPPORTED
    back = dict(q=3, r=w, br=1, codes=0x2000, ldc=2 ** 27 + 128, scales=0x3000, lds=3, dt=0, out=0x1000, ldo=w, stream=None)
    assert lib.lib().coded_f8_dequantize(*back.values()) == lib.CODED_ERR_UNSUPPORTED
    d = 2 ** 33 + 1
    assert lib.lib().coded_dropout(*{**DROP, "r": d, "ldx": d, "ldo": d}.values()) == lib.CODED_ERR_UNSUPPORTED
    assert lib.lib().coded_embed(*{**EMB, "d": d, "lde": d, "ldo": d}.values()) == lib.CODED_ERR_UNSUPPORTED
    assert lib.lib().coded_embed_grad(*{**GRAD, "d": d, "ldg": d, "ldde": d}.values()) == lib.CODED_ERR_UNSUPPORTED


@pytest.mark.parametrize("beta", [0.0, 1.0])
def test_gradients_of_more_parts_than_a_launch_joins(lib, beta):
    # 8192 tokens are 1024 chunks: 1023 joins of 2^24 / 512 pieces are more than a grid has, the sums before them are not
    d = 2 ** 24
    wide = {**GRAD, "n": 8192, "d": d, "ldg": d, "ldde": d, "beta": beta, "ws": 0x100000, "wsb": 2 ** 60}
    assert lib.lib().coded_embed_grad(*wide.values()) == lib.CODED_ERR_UNSUPPORTED


# ---------------------------------------------------------------- the binding

@pytest.fixture(scope="module")
def torch():
    return pytest.importorskip("torch")


def test_host_tensors_are_refused(lib, torch):
    """A host tensor would fault in a kernel: it is refused before any call."""
    x = torch.zeros(4, 4)
    M, MT = lib.alloc_f8(4, 4, device="cpu"), lib.alloc_f8(4, 4, device="cpu")
    tok = torch.zeros(4, dtype=torch.int64)
    for call in (lambda: lib.coded_f8_quantize(x, M, MT), lambda: lib.coded_f8_dequantize(M, x), lambda: lib.coded_f8_mm(M, MT, x),
                 lambda: lib.coded_dropout(x, x, 0.5, 1, 1), lambda: lib.coded_embed(x, tok, x.clone()), lambda: lib.coded_embed_grad(x, tok, x.clone())):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_binding_refuses_wrong_shapes(lib, torch):
    u8, f32 = torch.uint8, torch.float32
    good = lambda: (torch.zeros(5, 256, dtype=u8), torch.zeros(2, 5))
    lib.F8Matrix(*good(), 5, 200, 1)
    for codes, scales, rows, cols, block in [
            (torch.zeros(5, 200, dtype=u8), torch.zeros(2, 5), 5, 200, 1), (torch.zeros(4, 256, dtype=u8), torch.zeros(2, 5), 5, 200, 1),
            (torch.zeros(5, 256, dtype=u8), torch.zeros(1, 5), 5, 200, 1), (torch.zeros(5, 256, dtype=u8), torch.zeros(2, 4), 5, 200, 1),
            (torch.zeros(5, 256), torch.zeros(2, 5), 5, 200, 1), (torch.zeros(5, 256, dtype=u8), torch.zeros(2, 5, dtype=torch.float64), 5, 200, 1),
            (torch.zeros(256, 5, dtype=u8).t(), torch.zeros(2, 5), 5, 200, 1), (torch.zeros(5, 256, dtype=u8), torch.zeros(5, 2).t(), 5, 200, 1),
            (*good(), 5, 200, 2)]:
        with pytest.raises(ValueError):
            lib.F8Matrix(codes, scales, rows, cols, block)
    W = lib.alloc_f8(300, 200, 128, device="cpu")
    assert W.rows(128, 300).shape == (172, 200) and W.rows(128, 300).scales.shape == (2, 2)
    for a, b in ((1, 300), (128, 301), (256, 128)):
        with pytest.raises(ValueError):
            W.rows(a, b)
    x, tok = torch.zeros(5, 6), torch.zeros(5, dtype=torch.int64)
    A = lib.alloc_f8(5, 6, device="cpu")
    for call in (lambda: lib.coded_f8_quantize(x), lambda: lib.coded_f8_quantize(x, lib.alloc_f8(6, 5, device="cpu")),
                 lambda: lib.coded_f8_quantize(x, A, A), lambda: lib.coded_f8_quantize(x.half(), A), lambda: lib.coded_f8_dequantize(A, x.t()),
                 lambda: lib.coded_f8_mm(A, lib.alloc_f8(2, 7, device="cpu"), x), lambda: lib.coded_f8_mm(A, A, torch.zeros(5, 4)),
                 lambda: lib.coded_f8_mm(A, A, torch.zeros(5, 5), beta=1.0), lambda: lib.coded_f8_mm(A, A, torch.zeros(5, 5), beta=1.0, C=torch.zeros(4)),
                 lambda: lib.coded_dropout(x, x.bfloat16(), 0.5, 1, 1), lambda: lib.coded_dropout(x, x, 0.5, -1, 1), lambda: lib.coded_dropout(x, x, 0.5, 1, 1 << 56),
                 lambda: lib.coded_dropout(x, x, 0.5, 1, 1, C=x[:4]), lambda: lib.coded_embed(x, tok.int()[::2], torch.zeros(3, 6)),
                 lambda: lib.coded_embed(x, tok.float(), torch.zeros(5, 6)), lambda: lib.coded_embed(x, tok, torch.zeros(4, 6)),
                 lambda: lib.coded_embed_grad(x[:4], tok, x)):
        with pytest.raises(ValueError):
            call()


def test_a_workspace_must_be_as_long_as_its_elements_say(lib, torch):
    """An expanded tensor's elements are more than its memory; a kernel would write behind it."""
    one = torch.zeros(1, dtype=torch.uint8)
    A, X = lib.alloc_f8(300, 16384, 128, device="cpu"), lib.alloc_f8(260, 16384, device="cpu")
    M = lib.alloc_mx(16, 1 << 16, lib.CODED_MX4, device="cpu")
    tok, rows = torch.zeros(9, dtype=torch.int64), torch.zeros(9, 8)
    for ws in (one.expand(1 << 30), torch.zeros(1 << 20, 2, dtype=torch.uint8).t()):
        for call in (lambda: lib.coded_f8_mm(A, X, torch.zeros(300, 260), workspace=ws),
                     lambda: lib.coded_embed_grad(rows, tok, torch.zeros(20, 8), workspace=ws),
                     lambda: lib.coded_mx_mm(M, torch.zeros(1 << 16), torch.zeros(16), workspace=ws),
                     lambda: lib.coded_mx_mm_t(M, torch.zeros(16), torch.zeros(1 << 16), workspace=ws)):
            with pytest.raises(ValueError, match="contiguous"):
                call()
