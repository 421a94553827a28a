"""Dropout, embeddings and the way of a batch through them and an 8-bit layer, on the GPU, against the oracle in 64 bits."""
import numpy as np
import pytest

from oracle import f8 as of
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
    wide = np.full((a.shape[0], a.shape[1] + pad), np.nan, np.float32)
    wide[:, :a.shape[1]] = a
    return torch.from_numpy(wide).cuda().to(dtype)[:, :a.shape[1]]


HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def dt_of(torch, name):
    return torch.bfloat16 if name == "bf16" else torch.float32


# ---------------------------------------------------------------- dropout

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("q,r,p,first,pad", [(1, 1, 0.5, 0, 0), (3, 7, 0.1, 5, 1), (9, 8, 0.25, 0, 0), (5, 33, 0.9, (1 << 40) - 3, 3), (70, 129, 0.3, 1 << 33, 5), (2, 2100, 0.5, 1, 0)])
def test_dropout(lib, torch, q, r, p, first, pad, dtype, residual):
    rng = np.random.default_rng(q * 31 + r)
    dt = dt_of(torch, dtype)
    X = dense(torch, rng.standard_normal((q, r)), dt, pad)
    C = dense(torch, rng.standard_normal((q, r)), dt, pad) if residual else None
    wide = torch.full((q + 2, r + pad), 7.0, dtype=dt, device="cuda")
    out = wide[1:-1, :r]
    seed, draw = (1 << 64) - 5 - q, (1 << 56) - r
    lib.coded_dropout(X, out, p, seed, draw, first_row=first, C=C)
    kept = of.kept(q, r, p, seed, draw, first)
    x, c = host(X), host(C) if residual else 0.0
    want = np.where(kept, x / (1 - p), 0.0) + c
    # 1 / (1 - p), its product with x and the sum are rounded to fp32 at most once each, the result to its type
    bound = 2.0 ** -24 * (2 * np.abs(want - c) + np.abs(want)) * (1 + 2.0 ** -20) + HALF[dtype] * np.abs(want) * (1 + 2.0 ** -20)
    assert np.all(np.abs(host(out) - want) <= bound)
    if not residual:
        assert np.array_equal(host(out) != 0, kept & (x != 0))
    assert bool((wide[0] == 7).all()) and bool((wide[-1] == 7).all()) and bool((wide[:, r:] == 7).all())


def test_dropout_of_everything_and_nothing(lib, torch):
    x = torch.randn(5, 100, device="cuda")
    x[1, 3], x[2, 4] = float("nan"), float("inf")
    out = torch.full_like(x, 9.0)
    lib.coded_dropout(x, out, 1.0, 1, 1)
    assert bool((out == 0).all())
    lib.coded_dropout(x, out, 1.0, 1, 1, C=torch.ones_like(x))
    assert bool((out == 1).all())
    lib.coded_dropout(x, out, 0.0, 1, 1)
    assert torch.equal(out.nan_to_num(7), x.nan_to_num(7))
    for shape in ((0, 5), (5, 0)):
        lib.coded_dropout(torch.empty(shape, device="cuda"), torch.empty(shape, device="cuda"), 0.5, 1, 1)


def test_dropped_infinities_are_dropped(lib, torch):
    x = torch.full((8, 64), float("nan"), device="cuda")
    x[:, ::2] = float("inf")
    out = torch.empty_like(x)
    lib.coded_dropout(x, out, 0.5, 3, 4)
    assert np.array_equal(host(out) == 0, ~of.kept(8, 64, 0.5, 3, 4, 0))


def test_dropout_in_place_and_by_workers(lib, torch):
    x = torch.randn(301, 77, device="cuda")
    whole = torch.empty_like(x)
    lib.coded_dropout(x, whole, 0.3, 9, 2)
    parts = torch.empty_like(x)
    for a, b in ((0, 100), (100, 101), (101, 301)):
        lib.coded_dropout(x[a:b], parts[a:b], 0.3, 9, 2, first_row=a)
    assert torch.equal(whole, parts)
    y = x.clone()
    lib.coded_dropout(y, y, 0.3, 9, 2)
    assert torch.equal(y, whole)
    c = torch.randn_like(x)
    want = torch.empty_like(x)
    lib.coded_dropout(x, want, 0.3, 9, 2, C=c)
    lib.coded_dropout(x, c, 0.3, 9, 2, C=c)
    assert torch.equal(c, want)


def test_dropout_gradient_against_differences(lib, torch):
    """The map is linear, so its gradient is the same call: <D x, g> = <x, D g>, and a difference along any direction."""
    rng = np.random.default_rng(4)
    x, g = (torch.from_numpy(rng.integers(-8, 9, (40, 50)).astype(np.float32)).cuda() for _ in range(2))
    dx, dg = torch.empty_like(x), torch.empty_like(g)
    lib.coded_dropout(x, dx, 0.5, 1, 2)       # 1 / (1 - p) = 2: whole numbers throughout
    lib.coded_dropout(g, dg, 0.5, 1, 2)
    assert float((dx * g).sum()) == float((x * dg).sum())
    step = torch.zeros_like(x)
    step[3, 7] = step[20, 11] = 1.0
    up = torch.empty_like(x)
    lib.coded_dropout(x + step, up, 0.5, 1, 2)
    assert float(((up - dx) * g).sum()) == float((step * dg).sum())


# ---------------------------------------------------------------- embeddings

@pytest.mark.parametrize("e_dt", ["f32", "bf16"])
@pytest.mark.parametrize("o_dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,d,wide,pad", [(1, 1, 1, False, 0), (5, 10, 7, True, 1), (130, 33, 64, False, 3), (300, 1000, 129, True, 0), (40, 50, 2100, False, 1)])
def test_lookup(lib, torch, n, vocab, d, wide, pad, e_dt, o_dt):
    rng = np.random.default_rng(n + d)
    E = dense(torch, rng.standard_normal((vocab, d)), dt_of(torch, e_dt), pad)
    tok = rng.integers(0, vocab, n)
    skip = int(tok[0])
    if n > 4:
        tok[1], tok[2], tok[3] = -1, vocab, np.iinfo(np.int64 if wide else np.int32).min
    t = torch.from_numpy(tok.astype(np.int64 if wide else np.int32)).cuda()
    wide_out = torch.full((n + 2, d + pad), 7.0, dtype=dt_of(torch, o_dt), device="cuda")
    out = wide_out[1:-1, :d]
    lib.coded_embed(E, t, out, scale=1.7, skip=skip)
    want = of.embed(host(E), tok, 1.7, skip)
    got = host(out)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    fine = ~np.isnan(want)
    # the scale and the product are rounded to fp32, the result to its type
    assert np.all(np.abs(got - want)[fine] <= ((2.0 ** -23 + HALF[o_dt]) * (1 + 2.0 ** -8) * np.abs(want))[fine])
    assert bool((wide_out[0] == 7).all()) and bool((wide_out[-1] == 7).all()) and bool((wide_out[:, d:] == 7).all())


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("skip", [-1, 9, -100])
def test_a_skip_that_is_no_row_skips_none(lib, torch, skip, wide):
    """Tokens that the table lacks give NaN, also where skip is the same number; -1 is what a call without a skip has."""
    E = torch.arange(1.0, 9 * 20 + 1, device="cuda").view(9, 20)
    tok = torch.tensor([3, -1, 0, 9, 8, -100], dtype=torch.int64 if wide else torch.int32, device="cuda")
    for given in ({"skip": skip},) + (({},) if skip == -1 else ()):
        out = torch.zeros(6, 20, device="cuda")
        lib.coded_embed(E, tok, out, **given)
        assert torch.equal(out[[0, 2, 4]], E[[3, 0, 8]]) and bool(out[[1, 3, 5]].isnan().all())
        dE = torch.full_like(E, float("nan"))
        lib.coded_embed_grad(torch.ones(6, 20, device="cuda"), tok, dE, **given)
        want = torch.zeros_like(E)
        want[[3, 0, 8]] = 1.0
        assert torch.equal(dE, want)


def tokens_of(rng, kind, n, vocab):
    if kind == "same":
        return np.full(n, vocab // 2)
    if kind == "text":      # a few tokens make up much of it
        return np.minimum((np.exp(rng.random(n) * np.log(vocab + 1)) - 1).astype(np.int64), vocab - 1)
    tok = rng.integers(0, vocab, n)
    if kind == "bad" and n > 3:
        tok[rng.random(n) < 0.3] = -100
        tok[n // 2] = vocab + 5
    return tok


def check_gradient(lib, torch, kind, n, vocab, d, g_dt, e_dt, wide, beta, pad=0, whole=False):
    rng = np.random.default_rng(n * 3 + vocab + d)
    tok = tokens_of(rng, kind, n, vocab)
    skip = int(tok[0]) if kind == "bad" else -1
    G = dense(torch, rng.integers(-4, 5, (n, d)) if whole else rng.standard_normal((n, d)), dt_of(torch, g_dt), pad)
    t = torch.from_numpy(tok.astype(np.int64 if wide else np.int32)).cuda()
    wide_out = torch.full((vocab + 2, d + pad), 7.0, dtype=dt_of(torch, e_dt), device="cuda")
    dE = wide_out[1:-1, :d]
    old = host(dense(torch, rng.standard_normal((vocab, d)), dt_of(torch, e_dt)))
    dE.copy_(torch.from_numpy(old).cuda() if beta else torch.full((vocab, d), float("nan"), device="cuda"))
    scale = 2.0 if whole else 1.7
    lib.coded_embed_grad(G, t, dE, scale=scale, beta=beta, skip=skip)
    total, size, count = of.embed_grad(host(G), tok, vocab, skip)
    want = scale * total + (beta * old if beta else 0.0)
    got = host(dE)
    # m additions of fp32 numbers, m for the most frequent token; the scale, its product, and beta's
    m = count[:, None]
    bound = scale * (m + 4) * 2.0 ** -24 * size * (1 + 2.0 ** -10) + 2.0 ** -22 * np.abs(beta * old) + HALF[e_dt] * np.abs(want) * (1 + 2.0 ** -7)
    bound += HALF[e_dt] * (scale * (m + 4) * 2.0 ** -24 * size)
    if whole and not beta:
        assert np.array_equal(got, host(torch.from_numpy(want).to(dt_of(torch, e_dt))))
    else:
        assert np.all(np.abs(got - want) <= bound), np.max(np.abs(got - want) / np.maximum(bound, 1e-300))
    if beta == 1:
        none = count == 0
        assert np.array_equal(got[none], old[none])
    assert bool((wide_out[0] == 7).all()) and bool((wide_out[-1] == 7).all()) and bool((wide_out[:, d:] == 7).all())


@pytest.mark.parametrize("kind", ["any", "same", "text", "bad"])
@pytest.mark.parametrize("n,vocab,d", [(0, 5, 3), (1, 1, 1), (2, 3, 8), (63, 10, 9), (64, 200, 64), (65, 1, 130), (1000, 300, 33), (4096, 70, 8), (300, 5, 2100)])
def test_gradient_of_few_tokens(lib, torch, kind, n, vocab, d):
    if kind == "bad" and n == 0:
        kind = "any"
    check_gradient(lib, torch, kind, n, vocab, d, "f32", "f32", False, 0.0)
    check_gradient(lib, torch, kind, n, vocab, d, "bf16", "f32", True, 1.0, pad=1)


@pytest.mark.parametrize("g_dt", ["f32", "bf16"])
@pytest.mark.parametrize("e_dt", ["f32", "bf16"])
@pytest.mark.parametrize("beta", [0.0, 1.0, -0.5])
def test_gradient_of_any_type(lib, torch, g_dt, e_dt, beta):
    check_gradient(lib, torch, "bad", 500, 120, 40, g_dt, e_dt, True, beta, pad=3)
    check_gradient(lib, torch, "bad", 5000, 1200, 24, g_dt, e_dt, False, beta)


@pytest.mark.parametrize("kind", ["any", "same", "text", "bad"])
@pytest.mark.parametrize("n,vocab,d", [(4097, 100, 5), (10000, 511, 16), (10000, 512, 16), (70000, 3, 4), (300000, 300000, 3), (66000, 40000, 40)])
def test_gradient_of_many_tokens(lib, torch, kind, n, vocab, d):
    """Sorted in one, two and three digits, in one and many workgroups; whole numbers, so any lost or doubled row shows."""
    check_gradient(lib, torch, kind, n, vocab, d, "f32", "f32", n % 2 == 0, 0.0, whole=True)


def test_gradient_of_a_large_vocabulary(lib, torch):
    """Rows whose offsets pass 2^31 elements, tokens of 28 bits."""
    vocab, d = (1 << 28) + 3, 9
    dE = torch.zeros(vocab, d, dtype=torch.bfloat16, device="cuda")
    tok = torch.tensor([vocab - 1, 5, vocab - 1, 1 << 27] * 1500, dtype=torch.int32, device="cuda")
    G = torch.ones(6000, d, device="cuda")
    lib.coded_embed_grad(G, tok, dE, beta=1.0)
    # in bf16 a step is 16 at 3000 and 8 at 1500, and both are half way between two: 187.5 steps, 188 is even
    assert bool((dE[vocab - 1].float() == 3008).all()) and bool((dE[5].float() == 1504).all()) and bool((dE[1 << 27].float() == 1504).all())
    assert float(dE.sum(dtype=torch.float64)) == (3008 + 1504 + 1504) * d
    out = torch.empty(3, d, device="cuda")
    lib.coded_embed(dE, torch.tensor([vocab - 1, 0, vocab], device="cuda"), out)
    assert bool((out[0] == 3008).all()) and bool((out[1] == 0).all()) and bool(out[2].isnan().all())


def test_gradient_of_one_token_without_end(lib, torch):
    """2^24 rows of 1 + 2^-9 for one token.  A chunk's 64 rows, 512 chunks' sums in a wave's chain, 128 sums of those, and
    the four waves' bound the error by (64 + 513 + 128 + 4) 2^-24 of the sum; each chunk's sum after another, 65536 a
    wave, loses half a step 2^15 times in each: 2^-10."""
    n, d = 1 << 24, 3
    tok = torch.full((n,), 2, dtype=torch.int32, device="cuda")
    G = torch.full((n, d), 1 + 2.0 ** -9, device="cuda")
    dE = torch.empty(4, d, device="cuda")
    lib.coded_embed_grad(G, tok, dE)
    want = n * (1 + 2.0 ** -9)
    assert np.all(np.abs(host(dE)[2] - want) <= (64 + 513 + 128 + 4) * 2.0 ** -24 * want)
    assert bool((dE[[0, 1, 3]] == 0).all())


def test_gradient_is_the_same_every_time(lib, torch):
    rng = np.random.default_rng(0)
    tok = torch.from_numpy(tokens_of(rng, "text", 20000, 5000)).cuda()
    G = torch.randn(20000, 100, device="cuda")
    runs = []
    for _ in range(4):
        dE = torch.empty(5000, 100, device="cuda")
        lib.coded_embed_grad(G, tok, dE)
        runs.append(dE)
    assert all(torch.equal(runs[0], r) for r in runs[1:])


def test_gradient_is_the_transposed_lookup(lib, torch):
    """<E[tok], G> = <E, dE>, and a difference in a row of E; whole numbers."""
    rng = np.random.default_rng(7)
    E = torch.from_numpy(rng.integers(-5, 6, (50, 30)).astype(np.float32)).cuda()
    tok = torch.from_numpy(rng.integers(0, 50, 200)).cuda()
    G = torch.from_numpy(rng.integers(-5, 6, (200, 30)).astype(np.float32)).cuda()
    out, dE = torch.empty(200, 30, device="cuda"), torch.empty(50, 30, device="cuda")
    lib.coded_embed(E, tok, out, scale=3.0)
    lib.coded_embed_grad(G, tok, dE, scale=3.0)
    assert float((out * G).sum()) == float((E * dE).sum())
    step = E.clone()
    step[int(tok[0]), 4] += 1
    up = torch.empty_like(out)
    lib.coded_embed(step, tok, up, scale=3.0)
    assert float(((up - out) * G).sum()) == float(dE[int(tok[0]), 4])


# ---------------------------------------------------------------- together

class Layers:
    """tokens -> rows of a table -> dropout -> 8-bit layer, and back."""

    def __init__(self, lib, torch, n, vocab, r, q, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.lib, self.torch = lib, torch
        self.E = torch.randn(vocab, r, generator=g, device="cuda").bfloat16()
        self.tok = torch.randint(0, vocab, (n,), generator=g, device="cuda")
        self.dY = torch.randn(n, q, generator=g, device="cuda").bfloat16()
        W = torch.randn(q, r, generator=g, device="cuda") / r ** 0.5
        self.W, self.WT = lib.alloc_f8(q, r, 128), lib.alloc_f8(r, q, 128)
        lib.coded_f8_quantize(W, self.W, self.WT)
        self.X, self.XT = lib.alloc_f8(n, r), lib.alloc_f8(r, n)
        self.D, self.DT = lib.alloc_f8(n, q), lib.alloc_f8(q, n)
        empty = lambda *s, dt=torch.bfloat16: torch.empty(s, dtype=dt, device="cuda")
        self.rows, self.dropped, self.Y, self.dX = empty(n, r), empty(n, r), empty(n, q), empty(n, r)
        self.dW, self.dE = empty(q, r, dt=torch.float32), empty(vocab, r, dt=torch.float32)

    def step(self, stream=None):
        lib = self.lib
        lib.coded_embed(self.E, self.tok, self.rows, scale=2.0, stream=stream)
        lib.coded_dropout(self.rows, self.dropped, 0.25, 5, 6, stream=stream)
        lib.coded_f8_quantize(self.dropped, self.X, self.XT, stream=stream)
        lib.coded_f8_mm(self.W, self.X, self.Y, y_rows=True, stream=stream)
        lib.coded_f8_quantize(self.dY, self.D, self.DT, stream=stream)
        lib.coded_f8_mm(self.XT, self.DT, self.dW, y_rows=True, stream=stream)
        lib.coded_f8_mm(self.WT, self.D, self.dX, y_rows=True, stream=stream)
        lib.coded_dropout(self.dX, self.dX, 0.25, 5, 6, stream=stream)
        lib.coded_embed_grad(self.dX, self.tok, self.dE, scale=2.0, stream=stream)
        return [self.Y, self.dW, self.dX, self.dE]


@pytest.mark.parametrize("n,vocab,r,q", [(1, 7, 40, 30), (37, 11, 130, 150), (600, 500, 300, 260), (5000, 900, 136, 200)])
def test_a_training_step(lib, torch, n, vocab, r, q):
    """Every step against 64 bits from what the step before gave."""
    m = Layers(lib, torch, n, vocab, r, q)
    m.step()
    torch.cuda.synchronize()
    tok = m.tok.cpu().numpy()
    kept = of.kept(n, r, 0.25, 5, 6, 0)
    half = 2.0 ** -8 + 2.0 ** -22
    assert np.array_equal(host(m.rows), 2 * host(m.E)[tok])
    dropped = np.where(kept, host(m.rows) / 0.75, 0.0)
    assert np.all(np.abs(host(m.dropped) - dropped) <= half * np.abs(dropped))

    def stored(M):
        out = torch.empty(M.shape, device="cuda")
        lib.coded_f8_dequantize(M, out)
        return host(out)

    # codes are within half a step of what was stored, or half the smallest one
    for M, v in ((m.X, host(m.dropped)), (m.XT, host(m.dropped).T), (m.D, host(m.dY)), (m.DT, host(m.dY).T)):
        s = np.repeat(host(M.scales).T, 128, axis=1)[:, :M.cols]
        assert np.all(np.abs(stored(M) - v) <= (2.0 ** -4 + 2.0 ** -20) * np.abs(v) + s * 2.0 ** -10)
    W, WT, X, XT, D, DT = (stored(M) for M in (m.W, m.WT, m.X, m.XT, m.D, m.DT))
    assert np.array_equal(W, WT.T)
    for got, a, b, bf16 in ((m.Y, X, W, True), (m.dW, DT, XT, False)):
        want, size = a @ b.T, np.abs(a) @ np.abs(b).T
        bound = (192 + a.shape[1] / 128) * 2.0 ** -23 * size + 2.0 ** -21 * size
        if bf16:
            bound = bound + 7 * 2.0 ** -13 * size
            bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
        assert np.all(np.abs(host(got) - want) <= bound)
    dX, size = D @ WT.T, np.abs(D) @ np.abs(WT).T
    bound = (7 * 2.0 ** -13 + 2.0 ** -12) * size
    bound = bound + 2.0 ** -8 * (np.abs(dX) + bound)
    dX, bound = np.where(kept, dX / 0.75, 0.0), np.where(kept, bound / 0.75, 0.0)
    assert np.all(np.abs(host(m.dX) - dX) <= bound + half * (np.abs(dX) + bound))
    total, size, count = of.embed_grad(host(m.dX), tok, vocab, -1)
    assert np.all(np.abs(host(m.dE) - 2 * total) <= 2 * (count[:, None] + 4) * 2.0 ** -24 * size)


def test_two_captured_steps_and_an_eager_one(lib, torch):
    """Two graphs replayed in turn, each with workspaces of its own, between eager steps: every replay gives the eager result."""
    models = [Layers(lib, torch, 600, 500, 300, 260, seed=1), Layers(lib, torch, 4500, 700, 200, 140, seed=2)]
    want = [[t.clone() for t in m.step()] for m in models]
    torch.cuda.synchronize()
    graphs = []
    for m in models:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            m.step()
        graphs.append(g)
    eager = Layers(lib, torch, 600, 500, 300, 260, seed=1)
    for turn in range(4):
        for m in models:
            for t in (m.Y, m.dW, m.dX, m.dE):
                t.fill_(float("nan"))
        for g in graphs:
            g.replay()
        now = eager.step()
        torch.cuda.synchronize()
        for m, w in zip(models, want):
            assert all(torch.equal(t, v) for t, v in zip((m.Y, m.dW, m.dX, m.dE), w)), turn
        assert all(torch.equal(t, v) for t, v in zip(now, want[0]))
        # other tokens and gradients in the same places: the graphs read them anew
        for m in models + [eager]:
            m.tok.copy_((m.tok * 7 + turn) % m.E.shape[0])
        want = [[t.clone() for t in m.step()] for m in models]
        torch.cuda.synchronize()


def test_a_step_on_another_stream(lib, torch):
    m = Layers(lib, torch, 300, 100, 200, 150)
    want = [t.clone() for t in m.step()]
    torch.cuda.synchronize()
    for t in (m.Y, m.dW, m.dX, m.dE):
        t.fill_(float("nan"))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    m.step(stream=s)
    s.synchronize()
    assert all(torch.equal(t, w) for t, w in zip((m.Y, m.dW, m.dX, m.dE), want))
