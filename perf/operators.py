"""Microscaled formats on atom features and on what a network behind the grids keeps: what is timed.

Blocks of 32 numbers along a row share one power of two (the block and scale of the OCP Microscaling
Formats, v1.0); the elements are whole numbers of 8 bits, e4m3 or e2m1.  Four operators:

  keep      a tensor into codes and back, as a training step does with an activation between its
            forward and its backward pass (int8, e4m3) or a program with the matrices of a 4-bit
            product (e2m1).  Returns what the codes stand for.
  gradient  the weight gradient of a linear map of atom features, from the 8-bit codes of its input:
            dW[t,e] = sum over the atoms of G[m,t] X[m,e], db[t] = sum over the atoms of G[m,t].
            Atoms past ``natoms`` count for nothing, whatever their rows hold.
  product   two matrices in 4 bits: C = A B^T (+ bias), added up in float
  linear    the same with a left matrix in plain numbers, which the call takes to 4 bits itself: the
            map of atom features to channels where no gradient is wanted (screening), weights laid
            out once

A case has ``op``, ``format``, ``dtype`` (of the plain numbers), and sizes:
  keep      B N E: rows [B*N] of E (``flat``: the whole tensor is one row, as grids are kept)
  gradient  B N E T, ``ragged`` (examples of different length)
  product, linear   M N K, ``bias``

``run`` with ``own`` false is the plain form: blocks, comparisons and products of torch in float.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 32
TYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
SIZE = {"float32": 4, "float16": 2, "bfloat16": 2}
# element type: exponent of its largest number, largest number, significant bits below the leading
# one, exponent of its smallest normal number, significand past which the largest one rounds over
FORMATS = {"int8": (6, 127.0, None, None, 255 / 128),
           "e4m3": (8, 448.0, 3, -6, 29 / 16),
           "e2m1": (2, 6.0, 1, 0, 7 / 4)}


def listed():
    return [
        # ---- keep ----
        # the grids of a training batch (50 complexes, 28 channels, 48 points a side), kept by the
        # first layer behind them for its weight gradient: the largest tensor of the step
        dict(name="keep_grids", op="keep", format="int8", dtype="float32", B=50, N=28, E=110592,
             flat=True, values="grid"),
        # activations in half the resolution (24 points, 32 channels) of a network in bfloat16
        dict(name="keep_activations", op="keep", format="e4m3", dtype="bfloat16", B=50, N=32, E=13824,
             flat=True, values="relu"),
        # one small molecule's grid (4 channels, 24 points a side): latency
        dict(name="keep_small", op="keep", format="int8", dtype="float32", B=1, N=4, E=13824, flat=True,
             values="grid"),
        # features of the atoms of a batch of large complexes into 4 bits; odd rows
        dict(name="keep_features_4bit", op="keep", format="e2m1", dtype="float16", B=16, N=8000, E=509,
             flat=False, values="features"),
        # ---- gradient ----
        # learned types of a training batch: 50 complexes of 2040 atoms, 28 channels
        dict(name="gradient_batch", op="gradient", format="int8", dtype="float32", B=50, N=2040, E=256,
             T=28, ragged=False),
        # a batch of large complexes of different length, wide features, gradients in bfloat16
        dict(name="gradient_wide_ragged", op="gradient", format="e4m3", dtype="bfloat16", B=16, N=8000,
             E=1000, T=28, ragged=True),
        # one small molecule: latency
        dict(name="gradient_small", op="gradient", format="int8", dtype="float32", B=1, N=100, E=64, T=4,
             ragged=False),
        # ---- product ----
        # a wide hidden layer over the atoms of a batch: bound by the matrix cores
        dict(name="product_wide", op="product", format="e2m1", dtype="bfloat16", M=16320, N=4096, K=4096,
             bias=False),
        # one complex, odd sizes
        dict(name="product_odd", op="product", format="e2m1", dtype="float32", M=2040, N=509, K=1000,
             bias=True),
        # ---- linear ----
        # learned types of a screening batch: 50 complexes of 2040 atoms to 28 channels
        dict(name="linear_batch", op="linear", format="e2m1", dtype="float32", M=102000, N=28, K=256,
             bias=True),
        # a wide layer for a single row: the weights have to be read
        dict(name="linear_one_row", op="linear", format="e2m1", dtype="bfloat16", M=1, N=4096, K=4096,
             bias=False),
        # one small molecule: latency
        dict(name="linear_small", op="linear", format="e2m1", dtype="float16", M=100, N=28, K=256,
             bias=True),
    ]


def draw(rng):
    """One more case: sizes spread over the logarithm of their ranges, odd ones among them."""
    def span(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["keep", "gradient", "product", "linear"])
    dtype = rng.choice(list(TYPES))
    while True:
        if op == "keep":
            c = dict(op=op, format=rng.choice(list(FORMATS)), dtype=dtype, B=span(1, 64), N=span(4, 8000),
                     E=span(16, 20000), flat=rng.random() < 0.5,
                     values=rng.choice(["grid", "relu", "features"]))
            if 5e3 <= c["B"] * c["N"] * c["E"] <= 1.5e8:
                return c
        elif op == "gradient":
            c = dict(op=op, format=rng.choice(["int8", "e4m3"]), dtype=dtype, B=span(1, 64),
                     N=span(20, 8000), E=span(16, 1024), T=span(2, 128), ragged=rng.random() < 0.5)
            if c["B"] * c["N"] * c["E"] <= 1.3e8:
                return c
        else:
            c = dict(op=op, format="e2m1", dtype=dtype, M=span(1, 130000), N=span(4, 4096),
                     K=span(32, 4096), bias=rng.random() < 0.5)
            if 2.0 * c["M"] * c["N"] * c["K"] <= 5.4e11 and c["M"] * max(c["N"], c["K"]) <= 1.3e8:
                return c


# ---- the formats in plain torch ----

def _blocks(x):
    """[rows, cols] in float -> [rows, blocks, 32], the last block filled up with zeros."""
    rows, cols = x.shape
    n = (cols + BLOCK - 1) // BLOCK
    x = x.float()
    if n * BLOCK != cols:
        x = torch.nn.functional.pad(x, (0, n * BLOCK - cols))
    return x.reshape(rows, n, BLOCK)


def _shared(v, fmt):
    """The shared byte of every block: the smallest power of two for which the block's largest
    magnitude does not round past the largest element; 255 where the block is not finite."""
    emax, _, _, _, over = FORMATS[fmt]
    amax = v.abs().amax(dim=2)
    m, e = torch.frexp(amax)                                # amax = m 2^e, m in [1/2, 1)
    k = e - 1 + (2 * m >= over).int()
    s = (k - emax + 127).clamp(0, 254)
    s = torch.where(amax > 0, s, torch.zeros_like(s))
    return torch.where(torch.isfinite(amax), s, torch.full_like(s, 255))


def _power(s):
    """2^(s-127) in float (a power of two, so products with it are exact)."""
    return torch.pow(2.0, (s - 127).double()).float()


def _elements(v, s, fmt):
    """Numbers of the element type nearest to v 2^(127-s), ties to even, in float."""
    y = v * _power(254 - s)[..., None]
    y = torch.where((s == 255)[..., None], torch.zeros_like(y), y)
    _, top, bits, emin, _ = FORMATS[fmt]
    if fmt == "int8":
        return torch.round(y).clamp(-127, 127)
    _, e = torch.frexp(y)
    step = (((e - 1).clamp(min=emin) - bits + 127) << 23).view(torch.float32)      # a power of two, exactly
    return (torch.round(y / step) * step).clamp(-top, top)


def _values(el, s):
    """What elements and shared bytes stand for."""
    v = el * _power(s.clamp(max=254))[..., None]
    return torch.where((s == 255)[..., None], torch.full_like(v, math.nan), v)


def _quantised(x, fmt):
    """[rows, cols] -> the float values its codes stand for."""
    v = _blocks(x)
    s = _shared(v, fmt)
    return _values(_elements(v, s, fmt), s).reshape(x.shape[0], -1)[:, :x.shape[1]]


def _packed(x, fmt):
    """Codes and shared bytes as the library lays them out: a row of codes holds whole blocks (two
    e2m1 codes a byte, the even element in the low half), a row of shared bytes is filled up with
    zeros to a multiple of four."""
    v = _blocks(x)
    s = _shared(v, fmt)
    el = _elements(v, s, fmt).reshape(x.shape[0], -1)
    if fmt == "int8":
        codes = el.to(torch.int8).view(torch.uint8)
    elif fmt == "e4m3":
        codes = el.to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=x.device)
        codes = torch.bucketize(el.abs(), table).to(torch.uint8)
        codes = codes | (el < 0).to(torch.uint8) * 8
        codes = codes[:, 0::2] | (codes[:, 1::2] << 4)
    return codes.contiguous(), torch.nn.functional.pad(s.to(torch.uint8), (0, -s.shape[1] % 4))


def _unpacked(codes, scales, cols, fmt):
    """The float values of codes and shared bytes in that layout."""
    if fmt == "int8":
        el = codes.view(torch.int8).float()
    elif fmt == "e4m3":
        el = codes.view(torch.float8_e4m3fn).float()
    else:
        table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6],
                             device=codes.device)
        el = table[torch.stack([codes & 15, codes >> 4], dim=2).int()]
    el = el.reshape(codes.shape[0], -1, BLOCK)
    s = scales[:, :el.shape[1]].int()
    return _values(el, s).reshape(codes.shape[0], -1)[:, :cols]


# ---- inputs ----

def _natoms(c):
    """Atoms of every example: all of them, or (ragged) from a half on."""
    return [c["N"] - (37 * b * c["N"] // 64) % max(1, c["N"] // 2) if c["ragged"] else c["N"]
            for b in range(c["B"])]


def _numbers(shape, kind, dtype, g, dev):
    """grid: densities in [0, 2), most of space empty; relu: half of the numbers zero; features:
    normal, a scale of its own for every column (a few columns many times larger)."""
    x = torch.randn(shape, generator=g, device=dev)
    if kind == "grid":
        x = (0.6 * x.abs_()) * (torch.rand((shape[0], 1), generator=g, device=dev) + 0.3)
        patch = torch.rand((shape[0], (shape[1] + 95) // 96), generator=g, device=dev) < 0.4
        x *= patch.repeat_interleave(96, dim=1)[:, :shape[1]]
    elif kind == "relu":
        x = x.clamp_(min=0.0)
    else:
        col = torch.randn((shape[1],), generator=g, device=dev)
        x *= torch.exp(0.5 * col) * torch.where(col > 2.2, 8.0, 1.0)
    return x.to(dtype)


def prepare(case, seed):
    c = dict(case)
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed) * 6007 + 77)
    dtype = TYPES[c["dtype"]]
    s = {"case": c}
    if c["op"] == "keep":
        x = _numbers((c["B"] * c["N"], c["E"]), c["values"], dtype, g, dev)
        s["x"] = x.view(1, -1) if c["flat"] else x
    elif c["op"] == "gradient":
        x = _numbers((c["B"] * c["N"], c["E"]), "features", torch.float32, g, dev)
        G = (torch.randn((c["B"], c["N"], c["T"]), generator=g, device=dev) * 1e-3).to(dtype)
        s["natoms"] = None
        if c["ragged"]:
            s["natoms"] = torch.tensor(_natoms(c), dtype=torch.int32, device=dev)
            dead = torch.arange(c["N"], device=dev)[None, :] >= s["natoms"][:, None]
            x[dead.view(-1)] = math.nan         # nothing promises what the rows of no atom hold
            G[dead] = 0
        s["codes"], s["scales"] = _packed(x, c["format"])
        s["grad"] = G
    else:
        a = _numbers((c["M"], c["K"]), "features", dtype, g, dev)
        w = _numbers((c["N"], c["K"]), "features", torch.float32, g, dev) / math.sqrt(c["K"])
        s["w"] = _packed(w, c["format"])
        s["a"] = _packed(a, c["format"]) if c["op"] == "product" else a
        s["bias"] = torch.randn((c["N"],), generator=g, device=dev) if c["bias"] else None
    return s


# ---- one pass ----

def _own(s):
    from paper_1912_04822_amd import molgrid
    c = s["case"]
    dtype = TYPES[c["dtype"]]
    if c["op"] == "keep":
        return molgrid.mg_mx_unpack(molgrid.mg_mx_pack(s["x"], c["format"]))
    if c["op"] == "gradient":
        x = molgrid.MXTensor(s["codes"], s["scales"], (c["B"], c["N"], c["E"]), c["format"])
        return molgrid.mg_mx8_weight_gradient(s["grad"], x, natoms=s["natoms"])
    w = molgrid.MXTensor(*s["w"], (c["N"], c["K"]), c["format"])
    if c["op"] == "product":
        a = molgrid.MXTensor(*s["a"], (c["M"], c["K"]), c["format"])
        return molgrid.mg_mx4_product(a, w, bias=s["bias"], dtype=dtype)
    return molgrid.mg_mx4_linear(s["a"], w, bias=s["bias"])


def run(s):
    if own:
        return _own(s)
    c = s["case"]
    dtype = TYPES[c["dtype"]]
    if c["op"] == "keep":
        return _quantised(s["x"], c["format"]).to(dtype)
    if c["op"] == "gradient":
        x = _unpacked(s["codes"], s["scales"], c["E"], c["format"])
        G = s["grad"].float().view(-1, c["T"])
        if s["natoms"] is not None:
            dead = (torch.arange(c["N"], device=x.device)[None, :] >= s["natoms"][:, None]).view(-1, 1)
            x = torch.where(dead, torch.zeros_like(x), x)
            G = torch.where(dead, torch.zeros_like(G), G)
        return torch.matmul(G.t(), x), G.sum(dim=0)
    w = _unpacked(*s["w"], c["K"], c["format"])
    a = _unpacked(*s["a"], c["K"], c["format"]) if c["op"] == "product" else _quantised(s["a"], c["format"])
    y = torch.matmul(a, w.t())
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(dtype)


# ---- what a pass cannot do without ----

def work(case):
    c = case
    size = SIZE[c["dtype"]]
    code = (0.5 if c["format"] == "e2m1" else 1.0) + 1.0 / BLOCK
    if c["op"] == "keep":
        n = float(c["B"]) * c["N"] * c["E"]
        return {"bytes": 2.0 * n * (size + code), "flops": 4.0 * n}
    if c["op"] == "gradient":
        m = float(sum(_natoms(c)))
        return {"bytes": m * (c["T"] * size + c["E"] * code) + 4.0 * c["T"] * (c["E"] + 1),
                "flops": 2.0 * m * c["T"] * c["E"]}
    M, N, K = float(c["M"]), float(c["N"]), float(c["K"])
    left = M * K * (code if c["op"] == "product" else size)
    return {"bytes": left + N * K * code + M * N * size + (4 * N if c["bias"] else 0), "flops": 2 * M * N * K}


# ---- the same outputs in 64 bits, from the definition ----

def _levels(fmt):
    """The element type's numbers from zero up."""
    if fmt == "int8":
        return [float(q) for q in range(128)]
    if fmt == "e2m1":
        return [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    sub = [i * 2.0 ** -9 for i in range(8)]
    return (sub + [(8 + i) * 2.0 ** (e - 3) for e in range(-6, 9) for i in range(8)])[:-1]


def _two_to(e):
    """2^e in 64 bits, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _defined(x, fmt):
    """Every number goes to the nearest of the levels, by search; a tie goes to the level of even
    index (its last bit is zero)."""
    lv = torch.tensor(_levels(fmt), dtype=torch.float64, device=x.device)
    mid = (lv[1:] + lv[:-1]) / 2
    last = 2 * lv[-1] - mid[-1]                     # half a step above the largest level
    rows, cols = x.shape
    out = torch.empty((rows, cols), dtype=torch.float64, device=x.device)
    chunk = max(1, (1 << 25) // cols) if rows > 1 else 1
    width = cols if rows > 1 else 1 << 25           # a multiple of the block, or the whole row
    for r in range(0, rows, chunk):
        for q in range(0, cols, width):
            v = x[r:r + chunk, q:q + width].double()
            n = v.shape[1]
            v = torch.nn.functional.pad(v, (0, -n % 32)).unflatten(1, (-1, 32))
            amax = v.abs().amax(2, keepdim=True)
            k = torch.floor(torch.log2(amax)).nan_to_num(0, 0, -200).clamp(-200, 200)
            p = _two_to(k - FORMATS[fmt][0])
            p = torch.where(amax / p >= last, 2 * p, p).clamp(2.0 ** -127, 2.0 ** 127)
            a = v.abs() / p
            i = torch.searchsorted(mid, a.contiguous())             # mid[i-1] < a <= mid[i]
            tie = (i < len(mid)) & (a == mid[i.clamp(max=len(mid) - 1)]) & (i % 2 == 1)
            a = lv[i + tie.long()] * torch.sign(v) * p
            a = torch.where(torch.isfinite(amax), a, math.nan)
            out[r:r + chunk, q:q + width] = a.flatten(1)[:, :n]
    return out


def _stands_for(codes, scales, cols, fmt):
    """The numbers of stored codes: a table with an entry for each of them."""
    lv = _levels(fmt)
    if fmt == "int8":
        table = lv + [-128.0] + [-v for v in lv[:0:-1]]
    elif fmt == "e4m3":
        table = lv + [math.nan] + [-v for v in lv] + [math.nan]
    else:
        table = lv + [-v for v in lv]
        codes = torch.stack([codes % 16, codes // 16], -1).flatten(1)
    table = torch.tensor(table, dtype=torch.float64, device=codes.device)
    s = scales.repeat_interleave(32, dim=1)[:, :cols].double()
    v = table[codes[:, :cols].long()] * _two_to(s - 127)
    return torch.where(s == 255, math.nan, v)


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] == "keep":
        return _defined(s["x"], c["format"])
    if c["op"] == "gradient":
        x = _stands_for(s["codes"], s["scales"], c["E"], c["format"]).view(c["B"], c["N"], c["E"])
        G = s["grad"].double()
        dW = torch.zeros((c["T"], c["E"]), dtype=torch.float64, device=x.device)
        db = torch.zeros((c["T"],), dtype=torch.float64, device=x.device)
        for b, n in enumerate(_natoms(c)):
            dW += torch.matmul(G[b, :n].t().contiguous(), x[b, :n])
            db += G[b, :n].sum(0)
        return dW, db
    w = _stands_for(*s["w"], c["K"], c["format"])
    a = _stands_for(*s["a"], c["K"], c["format"]) if c["op"] == "product" else _defined(s["a"], c["format"])
    y = torch.matmul(a, w.t().contiguous())
    return y + s["bias"].double() if s["bias"] is not None else y
