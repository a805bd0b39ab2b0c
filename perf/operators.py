"""Performance cases of the operators on a vocabulary table.

The table W [V, d] is what a split head multiplies with and what the next
step's inputs are read from.  Four operators work on it:

  quantize   rows into microscaled 4-bit floating point, and the values that
             these stand for back again
  product    logits of hidden states against the kept rows of a table held in
             4 bits, the hidden states taken into the same format in `planes`
             terms (each term holds what the ones before it left over)
  lookup     a row of the table for each token, scaled
  gradient   the table's gradient from the gradients of the looked-up rows:
             the sum over a token's occurrences, for every row of the table

The 4-bit formats hold e2m1 codes (+-0, 0.5, 1, 1.5, 2, 3, 4, 6), two to a
byte, the even column in the low half, with a scale for each block of a row:

  e8m0   blocks of 32 columns; the scale is 2^(floor(log2(amax)) - 2), at
         least 2^-126, held as its exponent + 127
  e4m3   blocks of 16 columns; the scale is amax / 6 rounded to e4m3, in units
         of the row's own power of two, the least 2^k with amax(row) <= 2688 2^k

and x is coded as the e2m1 value nearest to x / scale (ties to the even code,
saturating at 6).

`prepare` gives what a program has in hand: hidden states as a slice of wider
rows, a table, the kept ids, tokens (frequent ids first, as tokenizers number
them), gradients.  `run` is one pass through the public calls; `exact` is the
definition in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
BLOCK = {"e8m0": 32, "e4m3": 16}
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}


def listed():
    return [
        # a decode head's table, 32000 x 4096, laid out in 4 bits once
        dict(name="quantize 32000x4096 bf16", kind="quantize", rows=32000, d=4096, fmt="e4m3",
             src="bf16"),
        # a few hidden states of an odd width, fp32: where a call's latency counts
        dict(name="quantize 5x1000 fp32", kind="quantize", rows=5, d=1000, fmt="e8m0", src="fp32"),
        # one decode row over a small subset: the tiny split head (d 512, d_l 64)
        dict(name="product 1x2048x448", kind="product", rows=1, V=8192, n=2048, d=448, d_l=64,
             fmt="e4m3", planes=2, h="fp32", out="fp32", bias=False),
        # 32 sessions' decode rows over a language subset (d 4096, d_l 256)
        dict(name="product 32x12000x3840", kind="product", rows=32, V=32000, n=12000, d=3840,
             d_l=256, fmt="e4m3", planes=2, h="fp32", out="fp32", bias=True),
        # 64 sessions x (4 drafts + 1) target rows over 40 % of the ids (d 4096, d_l 512)
        dict(name="product 320x51302x3584", kind="product", rows=320, V=128256, n=51302, d=3584,
             d_l=512, fmt="e4m3", planes=2, h="bf16", out="fp32", bias=False),
        # few rows over a whole large vocabulary (d 8192, d_l 1024), near-bf16 hidden states
        dict(name="product 8x152064x7168", kind="product", rows=8, V=152064, n=152064, d=7168,
             d_l=1024, fmt="e8m0", planes=3, h="fp32", out="fp32", bias=False),
        # many rows over the largest vocabulary (d 5120, d_l 512): the tensor-bound end
        dict(name="product 1024x256000x4608", kind="product", rows=1024, V=256000, n=256000,
             d=4608, d_l=512, fmt="e4m3", planes=1, h="bf16", out="bf16", bias=False),
        # the inputs of the next decode step of 32 sessions
        dict(name="lookup 32 of 32000x4096 bf16", kind="lookup", tokens=32, V=32000, d=4096,
             table="bf16", out="fp32", pad=0.0),
        # a batch of prompts through a table held in 4 bits, some of it padding
        dict(name="lookup 16384 of 256000x5120 e4m3", kind="lookup", tokens=16384, V=256000,
             d=5120, table="e4m3", out="bf16", pad=0.1),
        # a short adaptation step: the gradient of the whole table from 500 tokens
        dict(name="gradient 500 into 32000x4096", kind="gradient", tokens=500, V=32000, d=4096,
             src="fp32", out="fp32", pad=0.0, add=False),
        # a long one, whose frequent tokens occur thousands of times, into a large table
        dict(name="gradient 32768 into 128256x4096", kind="gradient", tokens=32768, V=128256,
             d=4096, src="bf16", out="bf16", pad=0.1, add=False),
        # added to the gradient that the table has already (from the head, where it is tied)
        dict(name="gradient 8000 onto 151643x3584", kind="gradient", tokens=8000, V=151643,
             d=3584, src="bf16", out="fp32", pad=0.0, add=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["quantize", "product", "product", "lookup", "gradient"])
    fmt = rng.choice(["e4m3", "e8m0"])
    if kind == "quantize":
        d = _log(rng, 17, 7168)
        return dict(kind=kind, rows=min(_log(rng, 1, 60000), 130000000 // d), d=d, fmt=fmt,
                    src=rng.choice(["bf16", "fp32", "fp16"]))
    if kind == "product":
        V = _log(rng, 500, 256000)
        n = V if rng.random() < 0.4 else max(1, int(V * rng.uniform(0.05, 0.9)))
        d, planes, out = _log(rng, 64, 4608), rng.choice([1, 2, 3, 4]), rng.choice(["fp32", "bf16"])
        most = min(int(1.2e12) // (n * d * planes), 524000000 // (n * SIZE[out]))
        return dict(kind=kind, rows=min(_log(rng, 1, 1000), most), V=V, n=n, d=d,
                    d_l=rng.choice([0, 48, 96, 129, 256, 512]), fmt=fmt, planes=planes,
                    h=rng.choice(["fp32", "bf16"]), out=out, bias=rng.random() < 0.3)
    V, d = _log(rng, 500, 200000), _log(rng, 32, 5120)
    V = min(V, 520000000 // d)
    if kind == "lookup":
        return dict(kind=kind, tokens=_log(rng, 1, 32768), V=V, d=d,
                    table=rng.choice(["bf16", "fp32", "e4m3", "e8m0"]),
                    out=rng.choice(["bf16", "fp32"]), pad=rng.choice([0.0, 0.2]))
    return dict(kind=kind, tokens=_log(rng, 1, 32768), V=V, d=d,
                src=rng.choice(["bf16", "fp32"]), out=rng.choice(["bf16", "fp32"]),
                pad=rng.choice([0.0, 0.2]), add=rng.random() < 0.3)


def _packed(rows, d, fmt):
    """Bytes of `rows` rows of d columns in 4 bits, with their scales."""
    return rows * (-(-d // 2) + -(-d // BLOCK[fmt]) + (4 if fmt == "e4m3" else 0))


def work(c):
    if c["kind"] == "quantize":
        n = c["rows"] * c["d"]
        return {"bytes": n * SIZE[c["src"]] + _packed(c["rows"], c["d"], c["fmt"]) + 2 * n,
                "flops": 4 * n}
    if c["kind"] == "product":
        b = _packed(c["n"], c["d"], c["fmt"]) + c["rows"] * c["d"] * SIZE[c["h"]]
        b += c["rows"] * c["n"] * SIZE[c["out"]] + (4 * c["n"] if c["n"] < c["V"] else 0)
        b += 4 * c["n"] if c["bias"] else 0
        return {"bytes": b, "flops": 2 * c["rows"] * c["n"] * c["d"]}
    T, V, d, out = c["tokens"], c["V"], c["d"], SIZE[c["out"]]
    distinct = _distinct(T * (1 - c["pad"]), V)
    if c["kind"] == "lookup":
        row = _packed(1, d, c["table"]) if c["table"] in BLOCK else d * SIZE[c["table"]]
        return {"bytes": 4 * T + distinct * row + T * d * out, "flops": T * d}
    rows = 2 * distinct if c["add"] else V
    return {"bytes": 4 * T + T * (1 - c["pad"]) * d * SIZE[c["src"]] + rows * d * out,
            "flops": T * (1 - c["pad"]) * d}


def _distinct(T, V):
    """Expected number of different ids among T tokens of _tokens()."""
    edges = [min(V, 2 ** k) for k in range(0, V.bit_length() + 1)]
    total, ln = 0.0, math.log(V + 1)
    for lo, hi in zip(edges, edges[1:]):
        if hi > lo:
            p = (math.log((hi + 1) / (lo + 1)) / ln) / (hi - lo)
            total += (hi - lo) * (1 - (1 - p) ** T)
    return total + 1 - (1 - math.log(2) / ln) ** T


# ---------------------------------------------------------------------------
# the inputs
# ---------------------------------------------------------------------------
_DEV = "cuda"


def _tokens(c, g):
    """Token ids with P(id) falling as 1 / (id + 1), a share of them the padding id -1."""
    V, T = c["V"], c["tokens"]
    u = torch.rand(T, generator=g, device=_DEV, dtype=torch.float64)
    t = (torch.exp(u * math.log(V + 1)) - 1).long().clamp_(0, V - 1).to(torch.int32)
    return torch.where(torch.rand(T, generator=g, device=_DEV) < c["pad"], -1, t).to(torch.int32)


def _pow2(k):
    """2^k in fp32 for whole k in [-126, 127]."""
    return ((k.int() + 127) << 23).view(torch.float32)


def _normal(shape, g, dtype, std=1.0):
    return torch.randn(shape, generator=g, device=_DEV, dtype=torch.float32).mul_(std).to(dtype)


def _table4(V, d, fmt, g):
    """A table of N(0, 0.02) weights in 4 bits: codes, scales and row scales as they are held."""
    bs, dp = BLOCK[fmt], -(-d // 32) * 32
    codes = torch.empty(V, dp // 2, dtype=torch.uint8, device=_DEV)
    scales = torch.zeros(V, -(-d // (16 * bs)) * 16, dtype=torch.uint8, device=_DEV)
    row = torch.ones(V, dtype=torch.float32, device=_DEV)
    step = max(1, (1 << 26) // dp)
    for a in range(0, V, step):
        x = _normal((min(V, a + step) - a, d), g, torch.float32, 0.02)
        q, s, r = _encode(x, fmt)
        code = _index(q)
        codes[a:a + step] = code[:, 0::2] | (code[:, 1::2] << 4)
        scales[a:a + step, :s.shape[1]] = _scale_bytes(s, fmt)
        row[a:a + step] = r[:, 0]
    return codes, scales, row if fmt == "e4m3" else None


def _index(q):
    """The 4-bit codes of e2m1 values: their place on the grid, bit 3 the sign."""
    a = q.abs()
    i = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4))
    return i.to(torch.uint8) | (torch.signbit(q).to(torch.uint8) << 3)


def _scale_bytes(s, fmt):
    if fmt == "e4m3":
        return s.to(torch.float8_e4m3fn).view(torch.uint8)
    return (torch.frexp(s)[1] + 126).to(torch.uint8)


def prepare(case, seed):
    c, g = case, torch.Generator(device=_DEV).manual_seed(seed)
    s = {"c": c}
    if c["kind"] == "quantize":
        # hidden states and weights alike: rows of different size, some channels far larger
        x = _normal((c["rows"], c["d"]), g, torch.float32)
        x *= torch.exp(_normal((c["rows"], 1), g, torch.float32))
        x[:, ::97] *= 20
        s["x"] = x.to(DTYPES[c["src"]])
    elif c["kind"] == "product":
        h = _normal((c["rows"], c["d_l"] + c["d"]), g, torch.float32)
        h /= h.square().mean(1, keepdim=True).sqrt()
        s["h"] = h.to(DTYPES[c["h"]])[:, c["d_l"]:]
        s["codes"], s["scales"], s["row_scale"] = _table4(c["V"], c["d"], c["fmt"], g)
        s["bias"] = _normal((c["V"],), g, torch.float32) if c["bias"] else None
        s["ids"] = _subset(c, g) if c["n"] < c["V"] else None
    elif c["kind"] == "lookup":
        s["tokens"] = _tokens(c, g)
        if c["table"] in BLOCK:
            s["codes"], s["scales"], s["row_scale"] = _table4(c["V"], c["d"], c["table"], g)
        else:
            s["table"] = _normal((c["V"], c["d"]), g, DTYPES[c["table"]], 0.02)
    else:
        s["tokens"] = _tokens(c, g)
        s["d_out"] = _normal((c["tokens"], c["d"]), g, DTYPES[c["src"]], 0.1)
        s["grad"] = _normal((c["V"], c["d"]), g, DTYPES[c["out"]]) if c["add"] else \
            torch.empty(c["V"], c["d"], dtype=DTYPES[c["out"]], device=_DEV)
    return s


def _subset(c, g):
    """Sorted kept ids in runs of 64 and more, as a language's ids lie in a vocabulary."""
    cell = 64
    cells = -(-c["V"] // cell)
    order = torch.rand(cells, generator=g, device=_DEV).argsort()
    first = order * cell
    ids = (first[:, None] + torch.arange(cell, device=_DEV)).reshape(-1)
    ids = ids[ids < c["V"]][:c["n"]]
    return ids.sort().values.to(torch.int32)


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
_ctx = None


def _context():
    global _ctx
    from paper_2607_13093_gb300 import sph
    if _ctx is None:
        _ctx = sph.Context(torch.cuda.current_device())
    return sph, _ctx


def _mx4(sph, s, fmt):
    return sph.Mx4(s["codes"], s["scales"], s["row_scale"], s["c"]["d"],
                   sph.SPH_MX4_E4M3 if fmt == "e4m3" else sph.SPH_MX4_E8M0)


def run(state):
    c = state["c"]
    if not own:
        return _PLAIN[c["kind"]](state, c)
    sph, ctx = _context()
    if c["kind"] == "quantize":
        fmt = sph.SPH_MX4_E4M3 if c["fmt"] == "e4m3" else sph.SPH_MX4_E8M0
        return ctx.mx4_dequantize(ctx.mx4_quantize(state["x"], fmt), dtype=torch.bfloat16)
    if c["kind"] == "product":
        return ctx.mx4_logits(state["h"], _mx4(sph, state, c["fmt"]), keep_ids=state["ids"],
                              bias=state["bias"], planes=c["planes"], dtype=DTYPES[c["out"]])
    if c["kind"] == "lookup":
        table = _mx4(sph, state, c["table"]) if c["table"] in BLOCK else state["table"]
        return ctx.embed(state["tokens"], table, scale=math.sqrt(c["d"]),
                         dtype=DTYPES[c["out"]])
    return ctx.embed_grad(state["tokens"], state["d_out"], c["V"], scale=math.sqrt(c["d"]),
                          accumulate=c["add"], out=state["grad"])


# ---- the plain form ---------------------------------------------------------
def _round_e2m1(a):
    """|values| to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6, ties to the even code."""
    q = 0.5 * (a > 0.25) + 0.5 * (a >= 0.75) + 0.5 * (a > 1.25) + 0.5 * (a >= 1.75)
    return q + 1.0 * (a > 2.5) + 1.0 * (a >= 3.5) + 2.0 * (a > 5.0)


def _encode(x, fmt):
    """fp32 rows [R, d] -> e2m1 values [R, dp], block scales [R, blocks], row scales [R, 1]."""
    R, d = x.shape
    bs, dp = BLOCK[fmt], -(-d // 32) * 32
    b = torch.nn.functional.pad(x, (0, dp - d)).view(R, dp // bs, bs)
    amax = b.abs().amax(2)
    row = torch.ones(R, 1, dtype=torch.float32, device=x.device)
    if fmt == "e4m3":
        m, e = torch.frexp(amax.amax(1, keepdim=True))
        row = torch.where(m > 0, _pow2((e - 12 + (m > 0.65625)).clamp(-110, 116)), row)
        s = (amax / torch.full_like(amax, 6.0) / row).to(torch.float8_e4m3fn).float()
    else:
        s = _pow2(torch.where(amax > 0, torch.frexp(amax)[1] - 3, -126).clamp(-126, 125))
    step = (s * row)[:, :, None]
    q = torch.copysign(_round_e2m1((b / step).abs().nan_to_num(0.0, 0.0)), b)
    return q.view(R, dp), s[:, :-(-d // bs)], row


def _values(q, s, row, fmt):
    """The values that codes and scales stand for, [R, dp]."""
    bs = BLOCK[fmt]
    s = torch.nn.functional.pad(s, (0, q.shape[1] // bs - s.shape[1]))
    return (q.view(q.shape[0], -1, bs) * s[:, :, None]).view(q.shape) * row


def _decode(codes, scales, row, d, fmt):
    """Held rows -> fp32 values [R, d]."""
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=codes.device)
    grid = torch.cat([grid, -grid])
    q = grid[torch.stack([codes & 15, codes >> 4], 2).view(codes.shape[0], -1).int()]
    s = scales[:, :-(-d // BLOCK[fmt])]
    s = s.contiguous().view(torch.float8_e4m3fn).float() if fmt == "e4m3" else \
        _pow2(s.int() - 127)
    one = torch.ones(1, 1, device=codes.device)
    return _values(q, s, one if row is None else row[:, None], fmt)[:, :d]


def _plain_quantize(s, c):
    q, scale, row = _encode(s["x"].float(), c["fmt"])
    return _values(q, scale, row, c["fmt"])[:, :c["d"]].to(torch.bfloat16)


def _terms(x, fmt, planes):
    """What `planes` 4-bit terms hold of x: each term codes what is left, in units of the first
    term's row scale."""
    d = x.shape[1]
    q, s, row = _encode(x, fmt)
    held = _values(q, s, row, fmt)[:, :d]
    for _ in range(planes - 1):
        held = held + _rest(x - held, row, fmt)
    return held


def _rest(x, row, fmt):
    """A later term: as _encode, with the row scale given."""
    R, d = x.shape
    if fmt == "e8m0":
        q, s, one = _encode(x, fmt)
        return _values(q, s, one, fmt)[:, :d]
    b = torch.nn.functional.pad(x, (0, -d % 32)).view(R, -1, 16)
    amax = b.abs().amax(2)
    s = (amax / torch.full_like(amax, 6.0) / row).to(torch.float8_e4m3fn).float()
    step = (s * row)[:, :, None]
    q = torch.copysign(_round_e2m1((b / step).abs().nan_to_num(0.0, 0.0)), b)
    return _values(q.view(R, -1), s, row, fmt)[:, :d]


def _plain_product(s, c):
    x = _terms(s["h"].float(), c["fmt"], c["planes"])
    if s["ids"] is None:
        held = s["codes"], s["scales"], s["row_scale"]
        bias = s["bias"]
    else:
        ids = s["ids"].long()
        held = s["codes"][ids], s["scales"][ids], None if s["row_scale"] is None else \
            s["row_scale"][ids]
        bias = None if s["bias"] is None else s["bias"][ids]
    y = x @ _decode(*held, c["d"], c["fmt"]).T
    return (y if bias is None else y + bias).to(DTYPES[c["out"]])


def _plain_lookup(s, c):
    t = s["tokens"].long()
    at = t.clamp(min=0)
    if c["table"] in BLOCK:
        row = None if s["row_scale"] is None else s["row_scale"][at]
        x = _decode(s["codes"][at], s["scales"][at], row, c["d"], c["table"])
    else:
        x = s["table"][at].float()
    x = x * torch.tensor(math.sqrt(c["d"]), dtype=torch.float32, device=x.device)
    return torch.where(t[:, None] >= 0, x, 0.0).to(DTYPES[c["out"]])


def _plain_gradient(s, c):
    t = s["tokens"].long()
    scale = torch.tensor(math.sqrt(c["d"]), dtype=torch.float32, device=t.device)
    total = torch.zeros(c["V"] + 1, c["d"], dtype=torch.float32, device=t.device)
    total.index_add_(0, torch.where(t < 0, c["V"], t), s["d_out"].float())
    total = total[:-1].mul_(scale)
    s["grad"].copy_(s["grad"].float() + total if c["add"] else total)
    return s["grad"]


_PLAIN = {"quantize": _plain_quantize, "product": _plain_product, "lookup": _plain_lookup,
          "gradient": _plain_gradient}


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------
_GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _nearest(a):
    """Grid value nearest to a >= 0 in 64 bits; of two equally near, the one of even index."""
    g = torch.tensor(_GRID, dtype=torch.float64, device=a.device)
    hi = torch.searchsorted(g, a.contiguous()).clamp(max=7)
    lo = (hi - 1).clamp(min=0)
    to_lo, to_hi = a - g[lo], g[hi] - a
    take_hi = (to_hi < to_lo) | ((to_hi == to_lo) & (hi % 2 == 0))
    return torch.where(take_hi, g[hi], g[lo])


def _two(k):
    """2^k in 64 bits."""
    return ((k.long() + 1023) << 52).view(torch.float64)


def _e4m3(v):
    """v >= 0 in 64 bits to the nearest e4m3 value (4 significant bits, least step 2^-9)."""
    unit = _two(torch.frexp(v)[1].clamp(min=-5) - 4)
    return torch.round(v / unit) * unit


def _terms64(x, fmt, planes):
    """sum of the terms of x (64 bits) in the given format."""
    R, d = x.shape
    bs = BLOCK[fmt]
    left = torch.nn.functional.pad(x, (0, -d % bs)).view(R, -1, bs)
    held = torch.zeros_like(left)
    top = left.abs().amax((1, 2))
    k = torch.where(top > 0, torch.ceil(torch.log2(top / 2688)), 0.0)
    k = torch.where(_two(k - 1) * 2688 >= top, k - 1, k)      # log2's own rounding
    k = torch.where(_two(k) * 2688 < top, k + 1, k)
    unit = torch.where(top > 0, _two(k.clamp(-110, 116)), 1.0)[:, None]
    for _ in range(planes):
        amax = left.abs().amax(2)
        if fmt == "e4m3":
            s = _e4m3(amax / (6 * unit)) * unit
        else:
            s = _two((torch.frexp(amax)[1] - 3).clamp(-126, 125))
        s = torch.where(amax > 0, s, 0.0)[:, :, None]
        q = _nearest(torch.where(s > 0, left.abs() / s, 0.0)) * s * torch.sign(left)
        held, left = held + q, left - q
    return held.view(R, -1)[:, :d]


def _table64(s, at, c, fmt):
    """Rows `at` (a slice or ids) of the held table in 64 bits."""
    codes, scales = s["codes"][at], s["scales"][at]
    g = torch.tensor(_GRID + [-v for v in _GRID], dtype=torch.float64, device=codes.device)
    q = torch.empty(codes.shape[0], 2 * codes.shape[1], dtype=torch.float64, device=codes.device)
    q[:, 0::2], q[:, 1::2] = g[(codes % 16).long()], g[(codes // 16).long()]
    b = scales.double()
    if fmt == "e4m3":
        e, m = torch.floor(b / 8), b % 8
        f = torch.where(e > 0, (1 + m / 8) * _two(e - 7), m / 8 * 2.0 ** -6)
        f = f * s["row_scale"][at].double()[:, None]
    else:
        f = _two(b - 127)
    return q[:, :c["d"]] * f.repeat_interleave(BLOCK[fmt], 1)[:, :c["d"]]


def exact(case, seed):
    c = case
    if c["kind"] == "product" and c["rows"] * c["n"] * c["d"] > 1.5e12:
        return None
    s = prepare(case, seed)
    if c["kind"] == "quantize":
        step = max(1, (1 << 25) // c["d"])
        return torch.cat([_terms64(s["x"][a:a + step].double(), c["fmt"], 1)
                          for a in range(0, c["rows"], step)])
    if c["kind"] == "product":
        x = _terms64(s["h"].double(), c["fmt"], c["planes"])
        ids = torch.arange(c["V"], device=x.device) if s["ids"] is None else s["ids"].long()
        y = torch.empty(c["rows"], c["n"], dtype=torch.float64, device=x.device)
        step = max(1, (1 << 27) // c["d"])
        for a in range(0, c["n"], step):
            y[:, a:a + step] = x @ _table64(s, ids[a:a + step], c, c["fmt"]).T
        return y if s["bias"] is None else y + s["bias"][ids].double()
    t = s["tokens"].long()
    # the scale is an fp32 argument of the call
    scale = float(torch.tensor(math.sqrt(c["d"]), dtype=torch.float32))
    if c["kind"] == "lookup":
        y = torch.zeros(c["tokens"], c["d"], dtype=torch.float64, device=t.device)
        kept = torch.nonzero(t >= 0)[:, 0]
        step = max(1, (1 << 26) // c["d"])
        for a in range(0, kept.numel(), step):
            k = kept[a:a + step]
            y[k] = scale * (_table64(s, t[k], c, c["table"]) if c["table"] in BLOCK else
                            s["table"][t[k]].double())
        return y
    y = torch.zeros(c["V"], c["d"], dtype=torch.float64, device=t.device)
    kept = torch.nonzero(t >= 0)[:, 0]
    y.index_add_(0, t[kept], s["d_out"][kept].double(), alpha=scale)
    return y + s["grad"].double() if c["add"] else y
