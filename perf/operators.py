"""The calls on microscaled 4-bit rows, as cases that can be timed and compared with their plain form.

Rows are held as blocks of 32 consecutive features that share a power of two (E8M0: byte s stands for 2^(s - 127), 255
for NaN); an element is E2M1: one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign.  A row of dim features has
B = ceil(dim / 32) blocks: codes [n][16 B] bytes (element 2 i of a block in the low half of byte i, the tail of the last
block zero) and scales [n][B] bytes.

  store    rows of some type are quantised and read back in that type (what a map with this kind of data does when
           it takes a batch in, and what its user looks at);
  load     stored rows are read back in some type;
  product  the dot products of all pairs of two sets of stored rows, in some type (an instance's response at every node);
  search   the nearest node of every stored row, the code book stored the same way (a trained map placing instances);
  epoch    ``Som.train_epoch`` on stored rows: the fp32 code book is quantised, searched, and updated from the rows' values.

``own`` = False computes them from elementary torch operations.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EPS_MASS = 1e-20


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # one instance arrives at a serving map of the common width: latency
        dict(name="store_one", op="store", n=1, dim=1_000, type="fp16"),
        # the training set of the many-instances configuration is taken in
        dict(name="store_set", op="store", n=1_000_000, dim=128, type="fp32"),
        # a page of a table looked at, odd in both sizes
        dict(name="load_page", op="load", n=777, dim=333, type="fp32"),
        # the whole training set of the headline configuration read back for another program
        dict(name="load_set", op="load", n=100_000, dim=1_000, type="bf16"),
        # one instance's response at every node of a 100 x 100 map
        dict(name="product_one", op="product", n=1, m=10_000, dim=128, type="fp32"),
        # responses of a batch at the nodes of a large map: what is written is what it costs
        dict(name="product_wide", op="product", n=50_000, m=10_000, dim=256, type="bf16"),
        # long rows such as embeddings, all pairs: what is computed is what it costs
        dict(name="product_long", op="product", n=8_192, m=8_192, dim=4_096, type="bf16"),
        # one instance placed on a trained 50 x 50 map: latency
        dict(name="search_one", op="search", n=1, k=2_500, dim=1_000),
        # the headline configuration's data placed on its map
        dict(name="search_set", op="search", n=100_000, k=2_500, dim=1_000),
        # the many-instances configuration: short rows, many nodes
        dict(name="search_large", op="search", n=1_000_000, k=10_000, dim=128),
        # a first run on a small table (configuration 1): every launch counts
        dict(name="epoch_toy", op="epoch", n=1_000, dim=10, rows=20, cols=20, radius=3.0),
        # an emergent map, about as many nodes as instances (configuration 3)
        dict(name="epoch_emergent", op="epoch", n=50_000, dim=256, rows=200, cols=200, radius=20.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    largest = {}
    for c in listed():
        w = work(c)
        for key in w:
            largest[c["op"], key] = max(largest.get((c["op"], key), 0), w[key])
    op = rng.choice(("store", "load", "product", "search", "epoch"))
    while True:
        dim = _log_int(rng, 10, 4_096)
        if op in ("store", "load"):
            c = dict(op=op, n=_log_int(rng, 1, 1_000_000), dim=dim, type=rng.choice(tuple(TYPES)))
        elif op == "product":
            c = dict(op=op, n=_log_int(rng, 1, 100_000), m=_log_int(rng, 1, 40_000), dim=dim, type=rng.choice(tuple(TYPES)))
        elif op == "search":
            c = dict(op=op, n=_log_int(rng, 1, 1_000_000), k=_log_int(rng, 1, 40_000), dim=dim)
        else:
            rows, cols = _log_int(rng, 5, 200), _log_int(rng, 5, 200)
            c = dict(op=op, n=_log_int(rng, 100, 200_000), dim=_log_int(rng, 10, 1_024), rows=rows, cols=cols,
                     radius=round(rng.uniform(0.1, 0.5) * min(rows, cols) + 1.0, 3))
        w = work(c)
        if all(w[key] <= largest[op, key] for key in w):
            return c


def _row_bytes(dim):
    return 17 * ((dim + 31) // 32)


def work(case):
    op, n, dim = case["op"], case["n"], case["dim"]
    rb = _row_bytes(dim)
    size = 4 if case.get("type", "fp32") == "fp32" else 2
    if op == "store":        # rows in, stored rows out; stored rows in, rows out
        return {"bytes": 2 * n * (dim * size + rb), "flops": 2 * n * dim}
    if op == "load":
        return {"bytes": n * (dim * size + rb), "flops": n * dim}
    if op == "product":
        return {"bytes": (n + case["m"]) * rb + n * case["m"] * size, "flops": 2 * n * case["m"] * dim}
    if op == "search":
        return {"bytes": (n + case["k"]) * rb + 4 * n, "flops": 2 * n * case["k"] * dim}
    k = case["rows"] * case["cols"]       # the sums' additions, two passes of the neighbourhood over the map
    return {"bytes": n * rb + 8 * k * dim + 4 * n,
            "flops": 2 * n * k * dim + n * dim + 2 * k * (case["rows"] + case["cols"]) * (dim + 1)}


# ---------------------------------------------------------------- inputs
def _clusters(n, dim, gen):
    """Rows around 64 centres with noise, features of different spread, as measured tables have them."""
    spread = torch.exp(0.7 * torch.randn(dim, generator=gen, device=DEV))
    centres = torch.randn(64, dim, generator=gen, device=DEV)
    which = torch.randint(0, 64, (n,), generator=gen, device=DEV)
    return (centres[which] + 0.3 * torch.randn(n, dim, generator=gen, device=DEV)) * spread


def _inputs(case, seed):
    """Tensors that the case starts from: what `run` and `exact` both compute on."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    op, n, dim = case["op"], case["n"], case["dim"]
    if op == "store":
        return {"rows": _clusters(n, dim, gen).to(TYPES[case["type"]])}
    if op == "load":
        return {"x": _plain_quantize(_clusters(n, dim, gen))}
    if op == "product":
        both = _clusters(n + case["m"], dim, gen)
        return {"x": _plain_quantize(both[:n]), "y": _plain_quantize(both[n:])}
    k = case["k"] if op == "search" else case["rows"] * case["cols"]
    both = _clusters(n + k, dim, gen)
    if op == "search":
        return {"x": _plain_quantize(both[:n]), "y": _plain_quantize(both[n:])}
    return {"x": _plain_quantize(both[:n]), "codebook": both[n:].contiguous()}


def prepare(case, seed):
    state = {"case": case, **_inputs(case, seed)}
    if own:
        from paper_1305_1422_amd import Mx4, Som
        for key in ("x", "y"):
            if key in state:
                state[key] = Mx4(*state[key])
        op = case["op"]
        if op == "epoch":
            state["som"] = Som(case["rows"], case["cols"], case["dim"], codebook=state["codebook"])
        elif op == "search":       # only the number of nodes counts: the code book is given in its stored form
            state["som"] = Som(1, case["k"], case["dim"], seed=1)
        else:
            state["som"] = Som(1, 1, case["dim"], seed=1)
    return state


# ---------------------------------------------------------------- one pass
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    case, som = state["case"], state["som"]
    op = case["op"]
    if op == "store":
        rows = state["rows"]
        return som.dequantize_mx4(som.quantize_mx4(rows), rows.dtype)
    if op == "load":
        return som.dequantize_mx4(state["x"], TYPES[case["type"]])
    if op == "product":
        return som.products_mx4(state["x"], state["y"], TYPES[case["type"]])
    if op == "search":
        return som.bmus(state["x"], nodes=state["y"])
    som.codebook.copy_(state["codebook"])
    bmus = som.train_epoch(state["x"], case["radius"])
    return bmus, som.codebook


def _run_plain(state):
    case = state["case"]
    op, dim = case["op"], case["dim"]
    if op == "store":
        rows = state["rows"]
        return _plain_values(_plain_quantize(rows), dim).to(rows.dtype)
    if op == "load":
        return _plain_values(state["x"], dim).to(TYPES[case["type"]])
    if op == "product":
        y = _plain_values(state["y"], dim).t()
        out = torch.empty((case["n"], case["m"]), dtype=TYPES[case["type"]], device=DEV)
        for lo in range(0, case["n"], 16_384):       # a table of 32-bit products at a time
            x = _plain_values([t[lo:lo + 16_384] for t in state["x"]], dim)
            out[lo:lo + 16_384] = torch.matmul(x, y)
        return out
    if op == "search":
        return _plain_search(state["x"], _plain_values(state["y"], dim), dim)
    codebook = state["codebook"]
    bmus = _plain_search(state["x"], _plain_values(_plain_quantize(codebook), dim), dim)
    return bmus, _plain_update(_plain_values(state["x"], dim), bmus, codebook, case["rows"], case["cols"], case["radius"])


# ---------------------------------------------------------------- plain forms
def _plain_quantize(rows):
    """(codes, scales) of rows [n][dim]: per block the power of two of its largest element, two down; nearest, ties to even."""
    n, dim = rows.shape
    blocks = (dim + 31) // 32
    codes, scales = [], []
    for lo in range(0, n, 131_072):
        x = rows[lo:lo + 131_072].float()
        m = x.shape[0]
        if dim != 32 * blocks:
            x = torch.cat([x, torch.zeros((m, 32 * blocks - dim), device=x.device)], 1)
        x = x.reshape(m, blocks, 32)
        size = x.abs()
        top = size.amax(2)
        s = torch.where(top > 0, torch.clamp(torch.frexp(top)[1] + 124, 0, 254), torch.zeros((), dtype=torch.int32, device=x.device))
        t = torch.ldexp(size, (127 - s).unsqueeze(2))
        q = ((t > 0.25).to(torch.uint8) + (t >= 0.75) + (t > 1.25) + (t >= 1.75) + (t > 2.5) + (t >= 3.5) + (t > 5.0)).to(torch.uint8)
        q = q | (torch.signbit(x).to(torch.uint8) << 3)
        codes.append((q[:, :, 0::2] | (q[:, :, 1::2] << 4)).reshape(m, 16 * blocks))
        scales.append(s.to(torch.uint8))
    return torch.cat(codes), torch.cat(scales)


def _plain_values(stored, dim):
    """The values that stored rows stand for, fp32 [n][dim]."""
    codes, scales = stored
    n, blocks = scales.shape
    level = torch.tensor(LEVELS + tuple(-v for v in LEVELS), dtype=torch.float32, device=codes.device)
    value = torch.empty((n, blocks, 32), dtype=torch.float32, device=codes.device)
    power = torch.ldexp(torch.ones((), device=codes.device), scales.to(torch.int32) - 127)
    power = torch.where(scales == 255, torch.full_like(power, math.nan), power).unsqueeze(2)
    packed = codes.reshape(n, blocks, 16)
    value[:, :, 0::2] = level[(packed & 15).int()] * power
    value[:, :, 1::2] = level[(packed >> 4).int()] * power
    return value.reshape(n, 32 * blocks)[:, :dim].contiguous()


def _plain_search(stored, nodes, dim):
    """Node of the largest x.w - |w|^2 / 2, in 64 bits: neighbouring nodes' scores lie close together, and equal ones occur."""
    w = nodes.double()
    half = 0.5 * (w * w).sum(1)
    index = torch.arange(w.shape[0], device=w.device, dtype=torch.int32)
    step = max(1, (1 << 27) // w.shape[0])
    found = []
    for lo in range(0, stored[0].shape[0], step):
        score = torch.matmul(_plain_values([t[lo:lo + step] for t in stored], dim).double(), w.t()) - half
        best = score.amax(1, keepdim=True)
        found.append(torch.where(score == best, index, w.shape[0]).amin(1))
    return torch.cat(found).to(torch.int32)


def _plain_update(values, bmus, codebook, rows, cols, radius):
    k, dim = codebook.shape
    sums = torch.zeros((k, dim), dtype=torch.float64, device=DEV).index_add_(0, bmus.long(), values.double())
    count = torch.zeros(k, dtype=torch.float64, device=DEV).index_add_(0, bmus.long(), torch.ones(bmus.shape[0], dtype=torch.float64, device=DEV))

    def weights(length):
        at = torch.arange(length, device=DEV, dtype=torch.float64)
        return torch.exp(-((at[:, None] - at[None, :]) ** 2) / (2.0 * radius * radius))

    image = torch.cat([sums, count[:, None]], 1)
    image = torch.matmul(weights(rows), image.reshape(rows, cols * (dim + 1)))
    image = image.reshape(rows, cols, dim + 1).transpose(0, 1).reshape(cols, rows * (dim + 1))
    image = torch.matmul(weights(cols), image).reshape(cols, rows, dim + 1).transpose(0, 1).reshape(k, dim + 1)
    mass = image[:, dim:]
    return torch.where(mass >= EPS_MASS, image[:, :dim] / mass, codebook.double()).float()


# ---------------------------------------------------------------- the definition in 64 bits
def _exact_values(stored, dim):
    codes, scales = stored
    low = codes.to(torch.int64)
    nibble = torch.stack([low % 16, low // 16], 2).reshape(codes.shape[0], -1)
    exponent, mantissa = (nibble // 2) % 4, nibble % 2
    size = torch.where(exponent == 0, 0.5 * mantissa.double(), (1.0 + 0.5 * mantissa.double()) * torch.pow(2.0, exponent.double() - 1.0))
    size = torch.where(nibble >= 8, -size, size)
    power = torch.pow(2.0, scales.double() - 127.0)
    power = torch.where(scales == 255, torch.full_like(power, math.nan), power)
    return (size * power.repeat_interleave(32, 1))[:, :dim]


def _exact_rounded(rows):
    """What rows are worth once stored: the nearest level of every element, of two equally near ones that with an even mantissa."""
    n, dim = rows.shape
    out = torch.empty((n, dim), dtype=torch.float64, device=DEV)
    order = (0.0, 1.0, 2.0, 4.0, 0.5, 1.5, 3.0, 6.0)          # even mantissas first: an equally near odd one does not replace them
    for lo in range(0, n, 65_536):
        x = rows[lo:lo + 65_536].double()
        for b in range(0, dim, 32):
            part = x[:, b:b + 32]
            top = part.abs().amax(1, keepdim=True)
            e = torch.where(top > 0, torch.clamp(torch.frexp(top)[1].double() - 3.0, -127.0, 127.0), torch.full_like(top, -127.0))
            scale = torch.pow(2.0, e)
            t = part.abs() / scale
            best, off = torch.zeros_like(t), t.clone()
            for v in order[1:]:
                d = (t - v).abs()
                best = torch.where(d < off, torch.full_like(t, v), best)
                off = torch.minimum(d, off)
            out[lo:lo + 65_536, b:b + 32] = torch.where(part < 0, -best, best) * scale
    return out


def _exact_nearest(x, w):
    """Lowest index of the smallest |w|^2 - 2 x.w; exact on values of this kind while their products span under 2^50."""
    norm = torch.square(w).sum(1)
    step = max(1, (1 << 26) // w.shape[0])
    wt = w.t().contiguous()
    out = torch.empty(x.shape[0], dtype=torch.int32, device=DEV)
    place = torch.arange(w.shape[0], 0, -1, device=DEV, dtype=torch.int32)
    for lo in range(0, x.shape[0], step):
        d = norm - 2.0 * torch.matmul(x[lo:lo + step], wt)
        least = d.min(1).values[:, None]
        out[lo:lo + step] = w.shape[0] - (place * (d <= least)).max(1).values
    return out


def exact(case, seed):
    given = _inputs(case, seed)
    op, dim = case["op"], case["dim"]
    if op == "store":
        return _exact_rounded(given["rows"])
    x = _exact_values(given["x"], dim)
    if op == "load":
        return x
    if op == "product":
        return torch.matmul(x, _exact_values(given["y"], dim).t().contiguous())
    if op == "search":
        return _exact_nearest(x, _exact_values(given["y"], dim))
    rows, cols, radius = case["rows"], case["cols"], case["radius"]
    codebook = given["codebook"].double()
    bmus = _exact_nearest(x, _exact_rounded(codebook))
    k = rows * cols
    order = torch.argsort(bmus.long(), stable=True)
    ends = torch.cumsum(torch.bincount(bmus.long(), minlength=k), 0)
    running = torch.cat([torch.zeros((1, dim), dtype=torch.float64, device=DEV), torch.cumsum(x[order], 0)])
    starts = torch.cat([torch.zeros(1, dtype=ends.dtype, device=DEV), ends[:-1]])
    sums, count = running[ends] - running[starts], (ends - starts).double()
    at_y = torch.div(torch.arange(k, device=DEV), cols, rounding_mode="floor").double()
    at_x = (torch.arange(k, device=DEV) % cols).double()
    out = torch.empty((k, dim), dtype=torch.float64, device=DEV)
    hit = torch.nonzero(count > 0).reshape(-1)
    sums, count = sums[hit], count[hit]
    for lo in range(0, k, 4_096):
        d2 = (at_y[lo:lo + 4_096, None] - at_y[hit]) ** 2 + (at_x[lo:lo + 4_096, None] - at_x[hit]) ** 2
        h = torch.exp(-d2 / (2.0 * radius * radius))
        mass = (h * count).sum(1, keepdim=True)
        out[lo:lo + 4_096] = torch.where(mass >= EPS_MASS, torch.matmul(h, sums) / mass, codebook[lo:lo + 4_096])
    return bmus, out
