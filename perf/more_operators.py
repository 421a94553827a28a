"""The way of a batch through the first layers of a model, as cases that can be run one by one.

Matrices in 8 bits hold E4M3 codes (up to 448) and an fp32 scale for each block
of 128 columns of a row, or of 128 x 128 (weights).  With m the largest
magnitude of a block, 2^-100 at least, the scale is m / 448, the factor u is
448 / m, both rounded to fp32, and a code is v u, rounded to fp32 and then to
the nearest code, ties to even.  The cases are

  store     a matrix as codes along its rows and, in the same pass, as codes
            along its columns (its transpose), both read back
  linear    Y = X W^T + bias: the batch X is stored in 8 bits, the weights W
            (128 x 128) are there in 8 bits; one token up to a whole batch
  backward  dX = dY W and dW = dY^T X + what there is: dY is stored both ways
            in one pass; W^T and X^T are there in 8 bits
  dropout   kept where a word of a counter-based generator says so, over 1 - p,
            plus a residual where there is one
  embed     rows of a table by tokens, scaled, and the gradient of the table
            from the gradient of those rows

A case is a dict of plain values.  linear: s tokens, q outputs, r features;
backward: s tokens, q outputs, r features too.  "pad" is how far rows of dense
inputs are apart beyond their length, in elements.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 128
TOP = 448.0
LEAST = 2.0 ** -100    # the smallest magnitude that a block's scale is made from
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
LARGEST_FLOPS = 2 * 16384 * 8192 * 8192


def listed():
    return [
        # Storing.  The published experiment's matrix, ends inside blocks both ways.
        _store("store_11500x5750", 11500, 5750, "f32"),
        # A batch of activations, 65536 tokens of 8192 features, for the forward and the backward pass.
        _store("store_65536x8192", 65536, 8192, "bf16"),
        # Forward.  One token through the smallest configured matrix: latency.
        _linear("linear_2048x512x1", 2048, 512, 1),
        # One token through the benchmark's default matrix.
        _linear("linear_65536x8192x1", 65536, 8192, 1),
        # A few tokens at once, ends inside blocks.
        _linear("linear_11500x5750x16", 11500, 5750, 16, x="f32", y="f32", bias=True),
        # A layer over a ragged batch.
        _linear("linear_16384x4096x4099", 16384, 4096, 4099, bias=True),
        # Backward.  The published matrix's shape and 10000 tokens: nothing is a multiple of a block.
        _backward("backward_11500x5750x10000", 11500, 5750, 10000),
        # A square layer over a large batch; the largest case.
        _backward("backward_8192x8192x16384", 8192, 8192, 16384),
        # Dropout.  The smallest configured matrix: launches alone.
        _dropout("dropout_2048x512", 2048, 512, "f32", 0.5),
        # The batch above after a layer, added to the residual.
        _dropout("dropout_65536x8192", 65536, 8192, "bf16", 0.1, residual=True),
        # Embedding.  A short prompt.
        _embed("embed_1000x512", 1000, 16384, 512, "f32"),
        # A batch of 65536 tokens; a word's frequency falls with its rank, as in text.
        _embed("embed_65536x4096", 65536, 65536, 4096, "bf16"),
    ]


def _store(name, q, r, dtype, pad=0):
    return {"name": name, "kind": "store", "q": q, "r": r, "dtype": dtype, "pad": pad}


def _linear(name, q, r, s, x="bf16", y="bf16", bias=False, pad=0):
    return {"name": name, "kind": "linear", "q": q, "r": r, "s": s, "x": x, "y": y, "bias": bias, "pad": pad}


def _backward(name, q, r, s, x="bf16", pad=0):
    return {"name": name, "kind": "backward", "q": q, "r": r, "s": s, "x": x, "pad": pad}


def _dropout(name, q, r, dtype, p, residual=False, first=0, pad=0):
    return {"name": name, "kind": "dropout", "q": q, "r": r, "dtype": dtype, "p": p, "residual": residual, "first": first, "pad": pad}


def _embed(name, n, vocab, d, dtype, pad=0, wide=False):
    return {"name": name, "kind": "embed", "n": n, "vocab": vocab, "d": d, "dtype": dtype, "pad": pad, "wide": wide}


def draw(rng):
    def spread(low, high):
        return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))

    kind = rng.choice(["store", "linear", "linear", "backward", "dropout", "embed"])
    dtype, pad = rng.choice(["f32", "bf16"]), rng.choice([0, 0, 1, 8])
    if kind == "store":
        q = spread(1, 131072)
        c = _store("", q, spread(1, min(16384, max(1, 65536 * 8192 // q))), dtype, pad)
    elif kind == "linear":
        q, r = spread(16, 65536), spread(16, 16384)
        # one token (serving) as often as a batch
        s = rng.choice([1, spread(2, 64), spread(65, 8192)])
        s = max(1, min(s, LARGEST_FLOPS // (2 * q * r), (1 << 29) // max(q, r)))
        c = _linear("", q, r, s, x=dtype, y=rng.choice(["f32", "bf16", "bf16"]), bias=rng.random() < 0.5, pad=pad)
    elif kind == "backward":
        q, r, s = spread(16, 16384), spread(16, 16384), spread(16, 16384)
        s = max(1, min(s, LARGEST_FLOPS // (4 * q * r)))
        c = _backward("", q, r, s, x=dtype, pad=pad)
    elif kind == "dropout":
        q = spread(1, 131072)
        c = _dropout("", q, spread(1, min(16384, max(1, 65536 * 8192 // q))), dtype, rng.choice([0.1, 0.25, 0.5]),
                     residual=rng.random() < 0.5, first=rng.choice([0, spread(1, 1 << 20)]), pad=pad)
    else:
        n, d = spread(1, 65536), spread(16, 4096)
        c = _embed("", n, spread(100, min(262144, (1 << 28) // d)), d, dtype, pad=pad, wide=rng.random() < 0.5)
    del c["name"]
    return c


# ---------------------------------------------------------------- inputs

def _generator(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 16 + stream) & ((1 << 62) - 1))
    return g


def _data(rows, cols, g, dtype=torch.float32, scale=1.0):
    """Normal values whose columns differ in size, as features do: one in 64 is eight times as large."""
    a = torch.randn((rows, cols), generator=g, device="cuda", dtype=torch.float32)
    size = torch.where(torch.rand(cols, generator=g, device="cuda") < 1 / 64, 8.0 * scale, scale)
    return (a * size).to(dtype)


def _strided(t, pad):
    """t in rows `pad` elements further apart than they are long."""
    if not pad:
        return t.contiguous()
    wide = torch.zeros((t.shape[0], t.shape[1] + pad), dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def _codes(a, block_rows):
    """(codes, one a byte, whole blocks of columns; scales, a row for every 128 columns) of a matrix in 8 bits."""
    q, r = a.shape
    v = torch.nn.functional.pad(a.to(torch.float32), (0, -r % BLOCK, 0, -q % block_rows))
    v = v.view(-1, block_rows, v.shape[1] // BLOCK, BLOCK)
    m = v.abs().amax((1, 3)).clamp(min=LEAST)
    top = torch.full_like(m, TOP)      # a division by or of a number would be a product with a reciprocal
    c = (v * (top / m)[:, None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    return c.view(-1, c.shape[2] * BLOCK)[:q], (m / top).t().contiguous()


def prepare(case, seed):
    g, kind = _generator(seed, 0), case["kind"]
    state = {"case": case}
    if kind == "store":
        # some tokens are padding: all zero
        a = _data(case["q"], case["r"], g, DT[case["dtype"]])
        a[torch.rand(case["q"], generator=g, device="cuda") < 1 / 16] = 0
        state["A"] = _strided(a, case["pad"])
    elif kind in ("linear", "backward"):
        q, r, s = case["q"], case["r"], case["s"]
        w = _data(q, r, g, scale=1 / 64)
        if kind == "linear":
            state["W"] = _codes(w, BLOCK)
            state["X"] = _strided(_data(s, r, _generator(seed, 1), DT[case["x"]]), case["pad"])
            if case["bias"]:
                state["bias"] = torch.randn(q, generator=_generator(seed, 2), device="cuda").to(DT[case["y"]])
        else:
            state["WT"] = _codes(w.t().contiguous(), BLOCK)
            state["XT"] = _codes(_data(s, r, _generator(seed, 1)).t().contiguous(), 1)
            state["dY"] = _strided(_data(s, q, _generator(seed, 2), DT[case["x"]], 1 / 256), case["pad"])
            state["dW"] = torch.randn((q, r), generator=_generator(seed, 3), device="cuda")
    elif kind == "dropout":
        q, r = case["q"], case["r"]
        state["X"] = _strided(_data(q, r, g, DT[case["dtype"]]), case["pad"])
        if case["residual"]:
            state["C"] = _data(q, r, _generator(seed, 1), DT[case["dtype"]])
        # a program's own seed, and how many masks it has drawn so far
        state["seed"], state["draw"] = (int(seed) * 0x9E3779B97F4A7C15 + 12345) % (1 << 64), int(seed) % 1000 + 7
    else:
        n, vocab, d = case["n"], case["vocab"], case["d"]
        state["E"] = torch.randn((vocab, d), generator=g, device="cuda").to(DT[case["dtype"]])
        # rank k of the vocabulary with a probability of about 1 / k
        rank = (torch.exp(torch.rand(n, generator=g, device="cuda", dtype=torch.float64) * math.log(vocab)) - 1).to(torch.int64)
        where = torch.randperm(vocab, generator=g, device="cuda")
        state["tokens"] = where[rank.clamp(0, vocab - 1)].to(torch.int64 if case["wide"] else torch.int32)
        state["G"] = _strided(_data(n, d, _generator(seed, 1), DT[case["dtype"]], 1 / 64), case["pad"])
    return state


# ---------------------------------------------------------------- one pass

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    from paper_1512_02673_amd import binding as lib
    case = state["case"]
    kind = case["kind"]
    if kind == "store":
        q, r = case["q"], case["r"]
        M, MT = lib.alloc_f8(q, r), lib.alloc_f8(r, q)
        lib.coded_f8_quantize(state["A"], M, MT)
        out = torch.empty((q, r), dtype=torch.bfloat16, device="cuda")
        out_t = torch.empty((r, q), dtype=torch.bfloat16, device="cuda")
        lib.coded_f8_dequantize(M, out)
        lib.coded_f8_dequantize(MT, out_t)
        return out, out_t
    if kind == "linear":
        q, r, s = case["q"], case["r"], case["s"]
        W = lib.F8Matrix(*state["W"], q, r, 128)
        X = lib.alloc_f8(s, r)
        lib.coded_f8_quantize(state["X"], X)
        Y = torch.empty((s, q), dtype=DT[case["y"]], device="cuda")
        lib.coded_f8_mm(W, X, Y, y_rows=True, beta=1.0 if case["bias"] else 0.0, C=state.get("bias"))
        return Y
    if kind == "backward":
        q, r, s = case["q"], case["r"], case["s"]
        WT, XT = lib.F8Matrix(*state["WT"], r, q, 128), lib.F8Matrix(*state["XT"], r, s, 1)
        D, DT_ = lib.alloc_f8(s, q), lib.alloc_f8(q, s)
        lib.coded_f8_quantize(state["dY"], D, DT_)
        dX = torch.empty((s, r), dtype=torch.bfloat16, device="cuda")
        dW = torch.empty((q, r), dtype=torch.float32, device="cuda")
        lib.coded_f8_mm(WT, D, dX, y_rows=True)
        lib.coded_f8_mm(XT, DT_, dW, y_rows=True, beta=1.0, C=state["dW"])
        return dX, dW
    if kind == "dropout":
        X = state["X"]
        out = torch.empty(X.shape, dtype=X.dtype, device="cuda")
        lib.coded_dropout(X, out, case["p"], state["seed"], state["draw"], first_row=case["first"], C=state.get("C"))
        return out
    E, G = state["E"], state["G"]
    out = torch.empty((case["n"], case["d"]), dtype=E.dtype, device="cuda")
    lib.coded_embed(E, state["tokens"], out, scale=case["d"] ** 0.5)
    dE = torch.empty(E.shape, dtype=torch.float32, device="cuda")
    lib.coded_embed_grad(G, state["tokens"], dE, scale=case["d"] ** 0.5)
    return out, dE


def _plain_values(codes, scales, cols, block_rows):
    """The fp32 matrix that codes and scales stand for."""
    v = codes.view(torch.float8_e4m3fn).to(torch.float32)
    rows = v.shape[0]
    per = scales.t() if block_rows == 1 else scales.t().repeat_interleave(block_rows, 0)[:rows]
    return (v.view(rows, -1, BLOCK) * per[:, :, None]).view(rows, -1)[:, :cols]


GAMMA, MIX1, MIX2 = (v - (1 << 64) if v >> 63 else v for v in (0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB))


def _mixed(z):
    """SplitMix64's output of a state, in wrapping 64-bit integers; the shifts bring in zeros."""
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * MIX1
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * MIX2
    return z ^ ((z >> 31) & ((1 << 33) - 1))


def _signed(v):
    v &= (1 << 64) - 1
    return v - (1 << 64) if v >> 63 else v


def _plain_kept(q, r, p, seed, number, first):
    """Which elements of rows first .. first + q - 1 are kept."""
    key = _mixed(torch.tensor(_signed(seed + ((10 << 56 | number) + 1) * GAMMA), device="cuda"))
    words = -(-r // 2)
    at = torch.arange(first * words, (first + q) * words, device="cuda").view(q, words)
    z = _mixed((at + 1) * GAMMA + key)
    halves = torch.stack((z & 0xFFFFFFFF, (z >> 32) & 0xFFFFFFFF), 2).view(q, 2 * words)[:, :r]
    return halves >= round(p * 2 ** 32)


def _run_plain(state):
    case = state["case"]
    kind = case["kind"]
    if kind == "store":
        q, r = case["q"], case["r"]
        A = state["A"].to(torch.float32)
        return (_plain_values(*_codes(A, 1), r, 1).to(torch.bfloat16), _plain_values(*_codes(A.t(), 1), q, 1).to(torch.bfloat16))
    if kind == "linear":
        r = case["r"]
        Y = _plain_values(*_codes(state["X"], 1), r, 1) @ _plain_values(*state["W"], r, BLOCK).t()
        if case["bias"]:
            Y = Y + state["bias"].to(torch.float32)
        return Y.to(DT[case["y"]])
    if kind == "backward":
        q, s = case["q"], case["s"]
        dY = state["dY"].to(torch.float32)
        dX = _plain_values(*_codes(dY, 1), q, 1) @ _plain_values(*state["WT"], q, BLOCK).t()
        dW = _plain_values(*_codes(dY.t(), 1), s, 1) @ _plain_values(*state["XT"], s, 1).t() + state["dW"]
        return dX.to(torch.bfloat16), dW
    if kind == "dropout":
        X = state["X"]
        kept = _plain_kept(case["q"], case["r"], case["p"], state["seed"], state["draw"], case["first"])
        out = torch.where(kept, X.to(torch.float32) * (1.0 / (1.0 - case["p"])), 0.0)
        if case["residual"]:
            out = out + state["C"].to(torch.float32)
        return out.to(X.dtype)
    tokens, scale = state["tokens"].to(torch.int64), case["d"] ** 0.5
    out = (state["E"][tokens].to(torch.float32) * scale).to(state["E"].dtype)
    dE = torch.zeros(state["E"].shape, dtype=torch.float32, device="cuda")
    dE.index_add_(0, tokens, state["G"].to(torch.float32))
    return out, dE * scale


# ---------------------------------------------------------------- in 64 bits

def _exact_values(codes, scales, cols, block_rows):
    """The matrix that codes and scales stand for, from the bits of each code."""
    c = codes.to(torch.int32)
    sign, e, m = c // 128, c // 8 % 16, c % 8
    v = torch.ldexp((m + torch.where(e > 0, 8, 0)).double(), (e.clamp(min=1) - 10).double())
    v = torch.where(sign == 1, -v, v)
    i = torch.arange(v.shape[0], device=v.device) // block_rows
    k = torch.arange(cols, device=v.device) // BLOCK
    return v[:, :cols] * scales.double()[k[None, :], i[:, None]]


def _exact_stored(a):
    """A matrix after it was stored, a row's blocks of 128 one by one."""
    out = torch.empty_like(a)
    for b in range(0, a.shape[1], BLOCK):
        v = a[:, b:b + BLOCK]
        m = v.abs().amax(1, keepdim=True).clamp(min=LEAST)
        u = (TOP / m).float().double()
        x = (v * u).float().double()
        _, e = torch.frexp(x)
        gap = torch.ldexp(torch.ones_like(x), ((e - 1).clamp(min=-6) - 3).double())     # between the codes around x
        out[:, b:b + BLOCK] = torch.round(x / gap) * gap * (m / TOP).float().double()
    return out


def _times(v, c):
    """v c modulo 2^64 for a constant c, from 32-bit halves of v (as two's complement numbers)."""
    lo, hi = v & 0xFFFFFFFF, (v >> 32) & 0xFFFFFFFF
    c0, c1 = c & 0xFFFFFFFF, c >> 32
    low = lo * (c0 & 0xFFFF) + ((lo * (c0 >> 16)) << 16)
    cross = (lo * (c1 & 0xFFFF) + hi * (c0 & 0xFFFF) + ((lo * (c1 >> 16) + hi * (c0 >> 16)) << 16)) & 0xFFFFFFFF
    return low + (cross << 32)


def _right(v, n):
    return torch.where(v < 0, (v >> n) + (1 << (64 - n)), v >> n)


def _exact_word(seed, number):
    """Output `number` (a tensor) of SplitMix64 seeded with `seed`."""
    z = _times(number + 1, 0x9E3779B97F4A7C15) + _signed(seed)
    z = _times(z ^ _right(z, 30), 0xBF58476D1CE4E5B9)
    z = _times(z ^ _right(z, 27), 0x94D049BB133111EB)
    return z ^ _right(z, 31)


def exact(case, seed):
    state = prepare(case, seed)
    kind = case["kind"]
    if kind == "store":
        A = state["A"].double()
        return _exact_stored(A), _exact_stored(A.t().contiguous())
    if kind == "linear":
        Y = torch.mm(_exact_stored(state["X"].double()), _exact_values(*state["W"], case["r"], BLOCK).t())
        return Y + state["bias"].double() if case["bias"] else Y
    if kind == "backward":
        dY = state["dY"].double()
        dX = torch.mm(_exact_stored(dY), _exact_values(*state["WT"], case["q"], BLOCK).t())
        dW = torch.mm(_exact_stored(dY.t().contiguous()), _exact_values(*state["XT"], case["s"], 1).t())
        return dX, dW + state["dW"].double()
    if kind == "dropout":
        q, r = case["q"], case["r"]
        key = int(_exact_word(state["seed"], torch.tensor(10 << 56 | state["draw"])))
        out = torch.zeros((q, r), dtype=torch.float64, device="cuda")
        words, step = -(-r // 2), max(1, (1 << 25) // r)
        for at in range(0, q, step):
            rows = torch.arange(case["first"] + at, case["first"] + min(q, at + step), device="cuda")
            w = _exact_word(key, rows[:, None] * words + torch.arange(words, device="cuda"))
            for odd in (0, 1):
                kept = (_right(w, 32) if odd else w % (1 << 32)) >= round(case["p"] * 2 ** 32)
                x = state["X"][at:at + step, odd::2].double()
                out[at:at + step, odd::2] = torch.where(kept[:, :x.shape[1]], x / (1 - case["p"]), 0.0)
        return out + state["C"].double() if case["residual"] else out
    tokens, scale = state["tokens"].to(torch.int64), math.sqrt(case["d"])
    order = torch.argsort(tokens, stable=True)
    values, count = torch.unique_consecutive(tokens[order], return_counts=True)
    dE = torch.zeros(state["E"].shape, dtype=torch.float64, device="cuda")
    step = 512      # columns at a time: sums of all the sorted rows so far, taken where a token ends
    end = torch.cumsum(count, 0) - 1
    for at in range(0, case["d"], step):
        upto = torch.cumsum(state["G"][:, at:at + step].double()[order], 0)[end]
        dE[values, at:at + step] = torch.diff(upto, dim=0, prepend=torch.zeros_like(upto[:1])) * scale
    return state["E"].double()[tokens] * scale, dE


def work(case):
    kind = case["kind"]
    if kind == "store":
        q, r = case["q"], case["r"]
        # read once, both sets of codes written, both read back as bf16; a product and two roundings each way
        return {"bytes": q * r * (SIZE[case["dtype"]] + 2 + 4), "flops": 6 * q * r}
    if kind == "linear":
        q, r, s = case["q"], case["r"], case["s"]
        return {"bytes": q * r + s * r * SIZE[case["x"]] + s * q * SIZE[case["y"]], "flops": 2 * q * r * s}
    if kind == "backward":
        q, r, s = case["q"], case["r"], case["s"]
        return {"bytes": q * r + s * r + s * q * SIZE[case["x"]] + 2 * s * r + 8 * q * r, "flops": 4 * q * r * s}
    if kind == "dropout":
        q, r = case["q"], case["r"]
        return {"bytes": q * r * SIZE[case["dtype"]] * (3 if case["residual"] else 2), "flops": 2 * q * r}
    n, vocab, d = case["n"], case["vocab"], case["d"]
    size = SIZE[case["dtype"]]
    # the rows that occur are read at most once; about as many as there are tokens in a short text
    return {"bytes": min(n, vocab) * d * size + 2 * n * d * size + vocab * d * 4, "flops": 2 * n * d}
