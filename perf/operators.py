"""Microscaled matrices: what a user has the library do with them, as cases that can be run one by one.

A microscaled matrix holds a row's values in blocks of 32 that share a power of
two: 4-bit codes (E2M1: 0, .5, 1, 1.5, 2, 3, 4, 6 with a sign) or 8-bit codes
(E4M3, up to 448), and one scale byte a block.  The cases are

  store  save a matrix as codes and read it back (weights in 4 bits, a batch of
         activations kept in 8 bits for the backward pass)
  mm     alpha A X + beta C, A microscaled, the sum along A's blocks (a worker's
         product, a layer's forward pass); X is fp32, bf16 or microscaled too
  mm_t   alpha A^T U + beta C, the sum across A's blocks (the second product of
         a gradient step, the gradient of a layer's input from its weights, the
         gradient of its weights from the saved batch)

A case is a dict of plain values: A is q x r of "bits", X (or U) and the result
have s columns.  "x_rows" and "y_rows" say that a right-hand side is a row of X
and of the result instead of a column; "pad" is how far X's rows are apart
beyond their length, in elements.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 32
LOWEST = 10            # the smallest scale byte that is written: 2^-117, so that every value is a normal bf16 number
TOP = {4: 6.0, 8: 448.0}
EMAX = {4: 2, 8: 8}    # exponent of the largest value of a format
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
LARGEST_FLOPS = 2 * 16384 * 8192 * 8192
LARGEST_A = 131072 * 16384


def listed():
    return [
        # Storing.  The smallest configured matrix: launches alone.
        _store("store4_2048x512", 2048, 512, 4, "f32"),
        # The published experiment's matrix, rows that end inside a block.
        _store("store4_11500x5750", 11500, 5750, 4, "f32"),
        # A batch of activations, 65536 tokens of 8192 features, kept for the backward pass.
        _store("store8_65536x8192", 65536, 8192, 8, "bf16"),
        # Products.  One vector through the smallest configured matrix: latency.
        _mm("mm4_2048x512x1", 2048, 512, 1),
        # One vector through the benchmark's default matrix: a worker's product,
        # or a single token through a large layer.
        _mm("mm4_65536x8192x1", 65536, 8192, 1),
        # A few right-hand sides, rows that end inside a block.
        _mm("mm4_11500x5750x16", 11500, 5750, 16, x="bf16"),
        # The dense workload's matrix and its 64 columns.
        _mm("mm4_131072x16384x64", 131072, 16384, 64, x="bf16"),
        # A layer's forward pass over a ragged batch of tokens, a token a row.
        _mm("mm4_16384x4096x4099", 16384, 4096, 4099, x="bf16", y="bf16", x_rows=True, y_rows=True),
        # The same with the batch in 8 bits, as it is saved; the largest case.
        _mm("mm4_16384x8192x8192_x8", 16384, 8192, 8192, x="mx8", y="bf16", x_rows=True, y_rows=True),
        # Transposed products.  The second half of a gradient step on the
        # configured least-squares problem: x - eta A^T z.
        _mm_t("mm_t4_262144x4096x1", 262144, 4096, 1, alpha=-0.5, beta=1.0),
        # The gradient of a layer's input from its 4-bit weights.
        _mm_t("mm_t4_16384x4096x4096", 16384, 4096, 4096, x="bf16", y="bf16", x_rows=True, y_rows=True),
        # The gradient of a layer's weights, of the published matrix's shape,
        # from the 8-bit batch of 10000 tokens; added to what there is.
        _mm_t("mm_t8_10000x5750x11500", 10000, 5750, 11500, bits=8, x="bf16", y_rows=True, beta=1.0),
    ]


def _store(name, q, r, bits, dtype):
    return {"name": name, "kind": "store", "q": q, "r": r, "bits": bits, "dtype": dtype, "pad": 0}


def _mm(name, q, r, s, bits=4, x="f32", y="f32", x_rows=False, y_rows=False, alpha=1.0, beta=0.0, pad=0, kind="mm"):
    return {"name": name, "kind": kind, "q": q, "r": r, "s": s, "bits": bits, "x": x, "y": y, "x_rows": x_rows,
            "y_rows": y_rows, "alpha": alpha, "beta": beta, "pad": pad}


def _mm_t(name, q, r, s, **more):
    return _mm(name, q, r, s, kind="mm_t", **more)


def draw(rng):
    def spread(low, high):
        return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))

    kind = rng.choice(["store", "mm", "mm", "mm_t"])
    if kind == "store":
        q = spread(1, 131072)
        r = spread(1, min(16384, max(1, 65536 * 8192 // q)))
        c = _store("", q, r, rng.choice([4, 8]), rng.choice(["f32", "bf16"]))
        c["pad"] = rng.choice([0, 0, 1, 8])
    else:
        q, r = spread(16, 262144), spread(16, 16384)
        q = max(1, min(q, LARGEST_A // r))
        # one right-hand side (serving, gradient steps) as often as a batch
        s = rng.choice([1, spread(2, 64), spread(65, 8192)])
        s = max(1, min(s, LARGEST_FLOPS // (2 * q * r)))
        # a result of at most a billion values
        s = max(1, min(s, (1 << 30) // max(q, r)))
        x = rng.choice(["f32", "bf16", "bf16", "mx8", "mx4"] if kind == "mm" else ["f32", "bf16", "bf16"])
        if x == "f32":   # three times a bf16 product's work
            s = max(1, min(s, LARGEST_FLOPS // (6 * q * r)))
        c = _mm("", q, r, s, bits=rng.choice([4, 4, 8]), x=x, y=rng.choice(["f32", "bf16"]),
                x_rows=x.startswith("mx") or rng.random() < 0.5, y_rows=rng.random() < 0.5, kind=kind,
                alpha=rng.choice([1.0, -0.5]), beta=rng.choice([0.0, 1.0]), pad=0 if x.startswith("mx") else rng.choice([0, 0, 1, 8]))
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


def _packed(rows, cols, bits, g, scale=1.0):
    """(codes, scales) of such a matrix, made a few rows at a time."""
    blocks = -(-cols // BLOCK)
    codes = torch.zeros((rows, blocks * BLOCK * bits // 8), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((rows, -(-blocks // 4) * 4), dtype=torch.uint8, device="cuda")
    size = torch.where(torch.rand(cols, generator=g, device="cuda") < 1 / 64, 8.0 * scale, scale)
    step = max(1, (1 << 26) // cols)
    for at in range(0, rows, step):
        end = min(rows, at + step)
        v = torch.randn((end - at, cols), generator=g, device="cuda") * size
        c, e = _codes(v, bits)
        codes[at:end] = c
        scales[at:end, :blocks] = e
    return codes, scales


def _codes(v, bits):
    """Code bytes and scale bytes of fp32 rows."""
    rows, cols = v.shape
    v = torch.nn.functional.pad(v, (0, -cols % BLOCK)).view(rows, -1, BLOCK)
    e = _scale_bytes(v, bits)
    scaled = v / (e << 23).view(torch.float32)[..., None]
    if bits == 8:
        c = scaled.clamp(-TOP[8], TOP[8]).to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        c = _e2m1(scaled)
        c = c[..., 0::2] | (c[..., 1::2] << 4)
    return c.reshape(rows, -1), e.to(torch.uint8)


def _scale_bytes(v, bits):
    """The biased exponent (int32) of each block's scale: the largest magnitude's exponent less the format's."""
    top = v.abs().amax(-1).contiguous()
    return ((top.view(torch.int32) >> 23) - EMAX[bits]).clamp(LOWEST, 254)


def _e2m1(a):
    """4-bit codes of scaled values, to nearest, ties to the even code."""
    m = a.abs()
    c = (m > 0.25).to(torch.uint8)
    for low, tie in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        c += (m >= low) if tie else (m > low)
    return c | (torch.signbit(a).to(torch.uint8) << 3)


def prepare(case, seed):
    g = _generator(seed, 0)
    q, r, bits = case["q"], case["r"], case["bits"]
    state = {"case": case}
    if case["kind"] == "store":
        # what is saved: weights or activations, some blocks of them all zero (padding tokens)
        a = _data(q, r, g, DT[case["dtype"]])
        a[torch.rand(q, generator=g, device="cuda") < 1 / 16] = 0
        state["A"] = _strided(a, case["pad"])
        return state
    s = case["s"]
    state["codes"], state["scales"] = _packed(q, r, bits, g, 1 / 64)
    k, n = (r, q) if case["kind"] == "mm" else (q, r)
    g = _generator(seed, 1)
    if case["x"].startswith("mx"):
        state["x_codes"], state["x_scales"] = _packed(s, k, int(case["x"][2:]), g)
    else:
        x = _data(s, k, g, DT[case["x"]])
        state["X"] = _strided(x if case["x_rows"] else x.t(), case["pad"])
    if case["beta"]:
        state["C"] = _data(*((s, n) if case["y_rows"] else (n, s)), _generator(seed, 2), DT[case["y"]])
    return state


# ---------------------------------------------------------------- one pass

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    from paper_1512_02673_amd import binding as lib
    case = state["case"]
    fmt = {4: lib.CODED_MX4, 8: lib.CODED_MX8}
    if case["kind"] == "store":
        A = state["A"]
        M = lib.alloc_mx(case["q"], case["r"], fmt[case["bits"]])
        lib.coded_mx_quantize(A, M)
        out = torch.empty((case["q"], case["r"]), dtype=torch.bfloat16, device="cuda")
        lib.coded_mx_dequantize(M, out)
        return out
    M = lib.MXMatrix(state["codes"], state["scales"], case["r"], fmt[case["bits"]])
    if "X" in state:
        X = state["X"]
    else:
        X = lib.MXMatrix(state["x_codes"], state["x_scales"], case["r"], fmt[int(case["x"][2:])])
    n = case["q"] if case["kind"] == "mm" else case["r"]
    Y = torch.empty((case["s"], n) if case["y_rows"] else (n, case["s"]), dtype=DT[case["y"]], device="cuda")
    call = lib.coded_mx_mm if case["kind"] == "mm" else lib.coded_mx_mm_t
    call(M, X, Y, x_rows=case["x_rows"], y_rows=case["y_rows"], alpha=case["alpha"], beta=case["beta"], C=state.get("C"))
    return Y


def _plain_values(codes, scales, cols, bits):
    """The fp32 matrix that codes and scales stand for."""
    rows = codes.shape[0]
    if bits == 8:
        v = codes.view(torch.float8_e4m3fn).to(torch.float32)
    else:
        table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=codes.device)
        v = table[torch.stack((codes & 15, codes >> 4), -1).view(rows, -1).to(torch.int32)]
    v = v.view(rows, -1, BLOCK)
    e = scales[:, :v.shape[1]].to(torch.int32)
    size = torch.where(e == 255, math.nan, (e << 23).view(torch.float32))
    return (v * size[..., None]).view(rows, -1)[:, :cols]


def _run_plain(state):
    case = state["case"]
    if case["kind"] == "store":
        rows, cols = state["A"].shape
        v = torch.nn.functional.pad(state["A"].to(torch.float32), (0, -cols % BLOCK)).view(rows, -1, BLOCK)
        top = v.abs().amax(-1).contiguous()
        size = (_scale_bytes(v, case["bits"]) << 23).view(torch.float32)
        size = torch.where(torch.isfinite(top), size, math.nan)[..., None]
        scaled = (v / size).clamp(-TOP[case["bits"]], TOP[case["bits"]])
        if case["bits"] == 8:
            scaled = scaled.to(torch.float8_e4m3fn).to(torch.float32)
        else:
            table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=v.device)
            scaled = table[_e2m1(scaled).to(torch.int32)]
        return (scaled * size).view(rows, -1)[:, :cols].to(torch.bfloat16)
    A = _plain_values(state["codes"], state["scales"], case["r"], case["bits"])
    if "X" in state:
        X = state["X"].to(torch.float32)
        X = X.t() if case["x_rows"] else X
    else:
        X = _plain_values(state["x_codes"], state["x_scales"], case["r"], int(case["x"][2:])).t()
    A = A if case["kind"] == "mm" else A.t()
    Y = (X.t() @ A.t() if case["y_rows"] else A @ X) * case["alpha"]
    if case["beta"]:
        Y = Y + case["beta"] * state["C"].to(torch.float32)
    return Y.to(DT[case["y"]])


# ---------------------------------------------------------------- in 64 bits

def _two_to(n):
    """2^n in 64 bits, from the bits of a float (n: whole numbers of a normal power)."""
    return ((n.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_values(codes, scales, cols, bits):
    """The matrix that codes and scales stand for, from the bits of each code."""
    c = codes.to(torch.int16)
    if bits == 4:
        c = torch.stack((c % 16, c // 16), 2).reshape(c.shape[0], -1)
    m_bits, e_bits = (1, 2) if bits == 4 else (3, 4)
    bias = 2 ** (e_bits - 1) - 1
    m, e, sign = c % 2 ** m_bits, c // 2 ** m_bits % 2 ** e_bits, c // 2 ** (m_bits + e_bits)
    v = (m + torch.where(e > 0, 2 ** m_bits, 0)).double() * _two_to(e.clamp(min=1) - bias - m_bits)
    v = torch.where(sign == 1, -v, v)
    per = torch.repeat_interleave(scales, BLOCK, 1)[:, :v.shape[1]].to(torch.int64)
    return (v * _two_to(per - 127))[:, :cols]


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "store":
        a, bits = state["A"].double(), case["bits"]
        q, r = a.shape
        out = torch.zeros((q, -(-r // BLOCK) * BLOCK), dtype=torch.float64, device=a.device)
        out[:, :r] = a
        out = out.reshape(q, -1, BLOCK)
        _, top = torch.frexp(out.abs().amax(2, keepdim=True))          # m = f 2^top with f in [1/2, 1)
        low = LOWEST - 127
        unit = torch.where(out.abs().amax(2, keepdim=True) > 0, top - 1 - EMAX[bits], low).clamp(min=low)
        v = out * _two_to(-unit)
        _, e = torch.frexp(v)
        # spacing of the codes around v: 2^(exponent - mantissa bits), no finer than the format's smallest value
        m_bits, least = (1, 0) if bits == 4 else (3, -6)
        gap = (e - 1).clamp(min=least) - m_bits
        v = (torch.round(v * _two_to(-gap)) * _two_to(gap)).clamp(-TOP[bits], TOP[bits])
        return (v * _two_to(unit)).reshape(q, -1)[:, :r]
    A = _exact_values(state["codes"], state["scales"], case["r"], case["bits"])
    if "X" in state:
        X = state["X"].double()
        X = X if case["x_rows"] else X.t().contiguous()
    else:
        X = _exact_values(state["x_codes"], state["x_scales"], case["r"], int(case["x"][2:]))
    Y = torch.mm(X, A.t() if case["kind"] == "mm" else A)              # a right-hand side a row
    Y = Y if case["y_rows"] else Y.t().contiguous()
    Y = case["alpha"] * Y
    return Y + case["beta"] * state["C"].double() if case["beta"] else Y


def work(case):
    q, r = case["q"], case["r"]
    blocks = -(-r // BLOCK)
    packed = q * (blocks * BLOCK * case["bits"] // 8 + blocks)
    if case["kind"] == "store":
        # read once, the codes and scales written, the values read back written; about a comparison, a product and a rounding each
        return {"bytes": q * r * (SIZE[case["dtype"]] + 2) + packed, "flops": 4 * q * r}
    s = case["s"]
    k, n = (r, q) if case["kind"] == "mm" else (q, r)
    x = s * (blocks * BLOCK * int(case["x"][2:]) // 8 + blocks) if case["x"].startswith("mx") else k * s * SIZE[case["x"]]
    y = n * s * SIZE[case["y"]] * (2 if case["beta"] else 1)
    return {"bytes": packed + x + y, "flops": 2 * q * r * s}
