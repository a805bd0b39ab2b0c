"""Performance cases of the operators around the head's product.

What a decoding or training step does with hidden states and logits next to
the product itself:

  norm       layer norm of hidden states, the last thing done to them before
             the head; `centre` false leaves the mean in
  grad       its backward pass: the gradient of its input, and those of weight
             and bias summed over all rows
  quantize   rows into e4m3 with an fp32 scale for each block of 128 columns of
             one row or of 128 rows, and the values that these stand for
  product    logits of hidden states, taken to e4m3 with a scale for each 128
             columns, against the kept rows of a table held so
  shape      logits with penalties for repeated tokens, biases and masks, and
             the token with the largest one

`prepare` gives what a program has in hand: hidden states (slices of wider rows
where it keeps them so), weights, a table, the kept ids, tokens so far, masks.
`run` is one pass through the public calls; `exact` is the definition in 64
bits.

Definitions beside the textbook ones:

  e4m3 block   scale = max(fp32(amax / 448), 2^-126); a code is the e4m3 value
               nearest to x / scale, ties to the even code
  shape        z, from a row's tokens so far (the first ones its prompt, the
               others its output) and per-row parameters:
               z / rep where z > 0, else z * rep, for ids among the tokens;
               z - freq * count, then z - pres, for ids among the output;
               z + the sum of the row's biases for the id;
               -inf where the row's mask has the id's bit clear
"""
from __future__ import annotations

import math

import torch

own = False

# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
EPS = 1e-5


def listed():
    return [
        # one decode row before the head: where a call's latency counts
        dict(name="norm 1x4096 bf16", kind="norm", rows=1, d=4096, x="bf16", out="fp32", wide=0,
             centre=False, bias=False),
        # a batch of prompts
        dict(name="norm 16384x5120 bf16", kind="norm", rows=16384, d=5120, x="bf16", out="bf16",
             wide=0, centre=True, bias=True),
        # a short adaptation step, fp32, an odd width that is a slice of wider rows
        dict(name="grad 500x4001 fp32", kind="grad", rows=500, d=4001, x="fp32", out="fp32",
             wide=95, centre=True, bias=True),
        # a long one in bf16
        dict(name="grad 32768x4096 bf16", kind="grad", rows=32768, d=4096, x="bf16", out="bf16",
             wide=0, centre=True, bias=True),
        # a few hidden states
        dict(name="quantize 5x1000 fp32", kind="quantize", rows=5, d=1000, block=1, x="fp32"),
        # a decode head's table, laid out once
        dict(name="quantize 32000x4096 bf16", kind="quantize", rows=32000, d=4096, block=128,
             x="bf16"),
        # one decode row over a small subset: the tiny split head (d 512, d_l 64)
        dict(name="product 1x2048x448", kind="product", rows=1, V=8192, n=2048, d=448, d_l=64,
             block=1, x="fp32", out="fp32", bias=False),
        # 32 sessions' decode rows over a language subset (d 4096, d_l 256)
        dict(name="product 32x12000x3840", kind="product", rows=32, V=32000, n=12000, d=3840,
             d_l=256, block=128, x="fp32", out="fp32", bias=True),
        # many rows over the largest vocabulary (d 5120, d_l 512): the tensor-bound end
        dict(name="product 1024x256000x4608", kind="product", rows=1024, V=256000, n=256000,
             d=4608, d_l=512, block=128, x="bf16", out="bf16", bias=False),
        # one decode row with a grammar and a long conversation behind it
        dict(name="shape 1x32000", kind="shape", rows=1, V=32000, n=32000, x="fp32", out="fp32",
             tokens=4000, biases=16, mask=True, penal=True, draw=True),
        # drafted target rows over a language subset, an odd number of ids
        dict(name="shape 320x51301", kind="shape", rows=320, V=128256, n=51301, x="fp32",
             out="fp32", tokens=1024, biases=0, mask=True, penal=True, draw=True),
        # many sessions over a whole vocabulary
        dict(name="shape 1024x128256", kind="shape", rows=1024, V=128256, n=128256, x="bf16",
             out="fp32", tokens=512, biases=64, mask=True, penal=True, draw=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "grad", "quantize", "product", "product", "shape", "shape"])
    types = ["bf16", "fp32", "fp16"]
    if kind in ("norm", "grad"):
        d = _log(rng, 33, 12000)
        return dict(kind=kind, rows=min(_log(rng, 1, 32768), 80000000 // d), d=d,
                    x=rng.choice(types), out=rng.choice(types), wide=rng.choice([0, 0, 8, 513]),
                    centre=rng.random() < 0.7, bias=rng.random() < 0.6)
    if kind == "quantize":
        d = _log(rng, 17, 7168)
        return dict(kind=kind, rows=min(_log(rng, 1, 60000), 130000000 // d), d=d,
                    block=rng.choice([1, 128]), x=rng.choice(types))
    V = _log(rng, 500, 256000)
    n = V if rng.random() < 0.4 else max(1, int(V * rng.uniform(0.05, 0.9)))
    if kind == "product":
        d, out = _log(rng, 64, 4608), rng.choice(["fp32", "bf16"])
        most = min(int(1.2e12) // (n * d), 524000000 // (n * SIZE[out]))
        return dict(kind=kind, rows=min(_log(rng, 1, 1000), most), V=V, n=n, d=d,
                    d_l=rng.choice([0, 48, 96, 129, 256, 512]), block=rng.choice([1, 128]),
                    x=rng.choice(["fp32", "bf16"]), out=out, bias=rng.random() < 0.3)
    penal = rng.random() < 0.8
    draws = rng.random() < 0.5
    return dict(kind=kind, rows=min(_log(rng, 1, 1024), 131000000 // n), V=V, n=n,
                x=rng.choice(["fp32", "bf16"]), out="fp32" if draws else rng.choice(["fp32", "bf16"]),
                tokens=_log(rng, 1, 8000) if penal else 0, biases=rng.choice([0, 3, 100]),
                mask=rng.random() < 0.6, penal=penal, draw=draws)


def work(c):
    R = c["rows"]
    if c["kind"] == "norm":
        n = R * c["d"]
        return {"bytes": n * (SIZE[c["x"]] + SIZE[c["out"]]) + 4 * c["d"] * (2 if c["bias"] else 1),
                "flops": 8 * n}
    if c["kind"] == "grad":
        n = R * c["d"]
        return {"bytes": n * (SIZE[c["x"]] + 2 * SIZE[c["out"]]) + 8 * R +
                4 * c["d"] * (3 if c["bias"] else 2), "flops": 16 * n}
    if c["kind"] == "quantize":
        n, blocks = R * c["d"], -(-c["d"] // 128)
        values = 4 if c["x"] == "fp32" else 2
        return {"bytes": n * (SIZE[c["x"]] + 1 + values) + 4 * blocks * -(-R // c["block"]),
                "flops": 4 * n}
    if c["kind"] == "product":
        n, d = c["n"], c["d"]
        scales = 4 * -(-d // 128) * -(-n // c["block"])
        b = n * d + scales + R * d * SIZE[c["x"]] + R * n * SIZE[c["out"]]
        b += (4 * n if n < c["V"] else 0) + (4 * n if c["bias"] else 0)
        return {"bytes": b, "flops": 2 * R * n * d}
    n = R * c["n"]
    b = n * (SIZE[c["x"]] + SIZE[c["out"]]) + 4 * R * c["tokens"] + 8 * R * c["biases"]
    b += R * c["n"] // 8 if c["mask"] else 0
    b += 4 * c["n"] if c["n"] < c["V"] else 0
    return {"bytes": b, "flops": 3 * n}


# ---------------------------------------------------------------------------
# the inputs
# ---------------------------------------------------------------------------
_DEV = "cuda"


def _normal(shape, g, dtype=torch.float32, std=1.0):
    return torch.randn(shape, generator=g, device=_DEV, dtype=torch.float32).mul_(std).to(dtype)


def _subset(V, n, g):
    """Sorted kept ids in runs of 64 and more, as a language's ids lie in a vocabulary."""
    cell = 64
    cells = -(-V // cell)
    first = torch.rand(cells, generator=g, device=_DEV).argsort() * cell
    ids = (first[:, None] + torch.arange(cell, device=_DEV)).reshape(-1)
    return ids[ids < V][:n].sort().values.to(torch.int32)


def _hidden(rows, d, g):
    """Hidden states: rows of different size, some channels far larger, a mean of their own."""
    x = _normal((rows, d), g)
    x *= torch.exp(_normal((rows, 1), g))
    x[:, ::97] *= 20
    return x.add_(_normal((rows, 1), g, std=0.3))


def prepare(case, seed):
    c, g = case, torch.Generator(device=_DEV).manual_seed(seed)
    s = {"c": c}
    R = c["rows"]
    if c["kind"] in ("norm", "grad"):
        d = c["d"]
        s["x"] = _hidden(R, d + c["wide"], g).to(DTYPES[c["x"]])[:, c["wide"]:]
        s["weight"] = _normal((d,), g, std=0.1).add_(1.0)
        s["bias"] = _normal((d,), g, std=0.1) if c["bias"] else None
        if c["kind"] == "grad":
            s["d_out"] = _normal((R, d), g, DTYPES[c["out"]], 0.1)
            # what the forward pass left
            x = s["x"].double()
            mean = x.mean(1, keepdim=True) if c["centre"] else torch.zeros_like(x[:, :1])
            var = (x - mean).square_().mean(1)
            s["mean"] = mean[:, 0].float() if c["centre"] else None
            s["rstd"] = (var + EPS).rsqrt().float()
    elif c["kind"] == "quantize":
        s["x"] = _hidden(R, c["d"], g).to(DTYPES[c["x"]])
    elif c["kind"] == "product":
        h = _normal((R, c["d_l"] + c["d"]), g)
        h /= h.square().mean(1, keepdim=True).sqrt()
        s["h"] = h.to(DTYPES[c["x"]])[:, c["d_l"]:]
        s["codes"], s["scales"] = _table8(c, g)
        s["bias"] = _normal((c["V"],), g) if c["bias"] else None
        s["ids"] = _subset(c["V"], c["n"], g) if c["n"] < c["V"] else None
    else:
        _prepare_shape(c, g, s)
    return s


def _table8(c, g):
    """A table of N(0, 0.02) weights in e4m3 with block scales, rows on 16 bytes."""
    V, d, block = c["V"], c["d"], c["block"]
    ld, kb = -(-d // 16) * 16, -(-d // 128)
    codes = torch.zeros(V, ld, dtype=torch.uint8, device=_DEV).view(torch.float8_e4m3fn)
    scales = torch.empty(-(-V // block), kb, dtype=torch.float32, device=_DEV)
    step = max(1, (1 << 26) // d // 128) * 128
    for a in range(0, V, step):
        x = _normal((min(V, a + step) - a, d), g, std=0.02)
        q, sc = _encode8(x, block)
        codes[a:a + step, :d] = q.to(torch.float8_e4m3fn)
        scales[a // block:a // block + sc.shape[0]] = sc
    return codes[:, :d], scales


def _prepare_shape(c, g, s):
    R, V, n, L = c["rows"], c["V"], c["n"], c["tokens"]
    s["ids"] = _subset(V, n, g) if n < V else None
    z = _normal((R, n), g, std=2.5)
    s["logits"] = z.to(DTYPES[c["x"]])
    s["tokens"] = s["lengths"] = s["prompts"] = s["rep"] = s["freq"] = s["pres"] = None
    if c["penal"]:
        # tokens so far: frequent ids first, as tokenizers number them, of different lengths
        u = torch.rand(R, L, generator=g, device=_DEV, dtype=torch.float64)
        s["tokens"] = (torch.exp(u * math.log(V + 1)) - 1).long().clamp_(0, V - 1).to(torch.int32)
        f = torch.rand(R, 2, generator=g, device=_DEV)
        s["lengths"] = (L * (0.5 + 0.5 * f[:, 0])).round().to(torch.int32)
        s["prompts"] = (s["lengths"] * f[:, 1]).to(torch.int32)
        s["rep"] = 1 + 0.3 * torch.rand(R, generator=g, device=_DEV)
        s["freq"] = 0.5 * torch.rand(R, generator=g, device=_DEV)
        s["pres"] = 0.5 * torch.rand(R, generator=g, device=_DEV)
    s["bias_ids"] = s["bias_values"] = s["mask"] = None
    if c["biases"]:
        # -1 stands for no entry: rows have lists of different lengths
        b = torch.randint(0, V, (R, c["biases"]), generator=g, device=_DEV, dtype=torch.int32)
        keep = torch.rand(R, c["biases"], generator=g, device=_DEV) < 0.9
        s["bias_ids"] = torch.where(keep, b, -1).to(torch.int32)
        s["bias_values"] = _normal((R, c["biases"]), g, std=3.0)
    if c["mask"]:
        # a grammar's masks: most rows allow a part of the ids, every fourth one all
        words = -(-V // 32)
        m = torch.randint(-2 ** 31, 2 ** 31, (3, R, words), generator=g, device=_DEV)
        m = torch.where((torch.arange(R, device=_DEV) % 4 == 3)[:, None], -1, m[0] & (m[1] | m[2]))
        s["mask"] = m.to(torch.int32)


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


def run(state):
    s, c = state, state["c"]
    if not own:
        return _PLAIN[c["kind"]](s, c)
    sph, ctx = _context()
    if c["kind"] == "norm":
        return ctx.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS, centre=c["centre"],
                              dtype=DTYPES[c["out"]])
    if c["kind"] == "grad":
        return ctx.layer_norm_grad(s["d_out"], s["x"], s["weight"], s["mean"], s["rstd"],
                                   bias=c["bias"], dtype=DTYPES[c["out"]])
    if c["kind"] == "quantize":
        w = ctx.fp8_quantize(s["x"], c["block"])
        return ctx.fp8_dequantize(w, dtype=_values_type(c))
    if c["kind"] == "product":
        return ctx.fp8_logits(s["h"], sph.Fp8(s["codes"], s["scales"], c["block"]),
                              keep_ids=s["ids"], bias=s["bias"], dtype=DTYPES[c["out"]])
    return ctx.shape_logits(s["logits"], c["V"], keep_ids=s["ids"], history=s["tokens"],
                            lengths=s["lengths"], prompt_lengths=s["prompts"],
                            repetition=s["rep"], frequency=s["freq"], presence=s["pres"],
                            bias_ids=s["bias_ids"], bias_values=s["bias_values"], mask=s["mask"],
                            temperature=0.0 if c["draw"] else None, dtype=DTYPES[c["out"]])


def _values_type(c):
    return torch.float32 if c["x"] == "fp32" else torch.bfloat16


def _two(k):
    """2^k in 64 bits."""
    return ((k.long() + 1023) << 52).view(torch.float64)


# ---- the plain form ---------------------------------------------------------
def _plain_norm(s, c):
    x = s["x"].float()
    if c["centre"]:
        x = x - x.mean(1, keepdim=True)
    y = x * torch.rsqrt(x.square().mean(1, keepdim=True) + EPS) * s["weight"]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(DTYPES[c["out"]])


def _plain_grad(s, c):
    x, dy = s["x"].float(), s["d_out"].float()
    r = s["rstd"][:, None]
    xh = (x - s["mean"][:, None] if c["centre"] else x) * r
    g = dy * s["weight"]
    dx = g - xh * (g * xh).mean(1, keepdim=True)
    if c["centre"]:
        dx = dx - g.mean(1, keepdim=True)
    dw = (dy * xh).sum(0)
    return (dx * r).to(DTYPES[c["out"]]), dw, dy.sum(0) if c["bias"] else None


def _blocks(x, block):
    """[R, d] -> [rows of blocks, block, column blocks, 128], zeros where there is nothing."""
    R, d = x.shape
    x = torch.nn.functional.pad(x, (0, -d % 128, 0, -R % block))
    return x.view(-1, block, x.shape[1] // 128, 128)


def _encode8(x, block):
    """fp32 rows -> e4m3 values (fp32) [R, d] and block scales.  Quotients and their rounding in
    64 bits: in 32 a quotient can round onto the border of two codes."""
    b = _blocks(x, block)
    amax = b.abs().amax((1, 3))
    scales = (amax / torch.full_like(amax, 448.0)).clamp(min=2.0 ** -126)
    t = b.double() / scales.double()[:, None, :, None]
    unit = _two(torch.frexp(t)[1].clamp(min=-5) - 4)
    q = (torch.round(t / unit) * unit).float()
    return q.reshape(-1, q.shape[2] * 128)[:x.shape[0], :x.shape[1]], scales


def _decode8(q, scales, block, d, at=None):
    """e4m3 codes [R, d] of rows `at` (None: all, in order) -> their fp32 values."""
    rows = torch.arange(q.shape[0], device=q.device) if at is None else at
    f = scales[torch.div(rows, block, rounding_mode="floor")]
    return q.float() * f.repeat_interleave(128, 1)[:, :d]


def _plain_quantize(s, c):
    out = torch.empty(c["rows"], c["d"], dtype=_values_type(c), device=s["x"].device)
    step = max(1, (1 << 25) // c["d"] // 128) * 128
    for a in range(0, c["rows"], step):
        q, scales = _encode8(s["x"][a:a + step].float(), c["block"])
        out[a:a + step] = _decode8(q, scales, c["block"], c["d"]).to(out.dtype)
    return out


def _plain_product(s, c):
    q, sx = _encode8(s["h"].float(), 1)
    x = _decode8(q, sx, 1, c["d"])
    ids = s["ids"].long() if s["ids"] is not None else None
    codes = s["codes"] if ids is None else s["codes"].view(torch.uint8)[ids].view(torch.float8_e4m3fn)
    y = x @ _decode8(codes, s["scales"], c["block"], c["d"], ids).T
    if s["bias"] is not None:
        y = y + (s["bias"] if ids is None else s["bias"][ids])
    return y.to(DTYPES[c["out"]])


def _counts(s, c):
    """How often each id [R, V] is among the prompt's and the output's tokens."""
    t = s["tokens"].long()
    at = torch.arange(t.shape[1], device=t.device)[None]
    prompt = at < s["prompts"][:, None]
    there = at < s["lengths"][:, None]
    out = []
    for part in (there & prompt, there & ~prompt):
        n = torch.zeros(t.shape[0], c["V"], dtype=torch.int32, device=t.device)
        out.append(n.scatter_add_(1, t, part.to(torch.int32)))
    return out


def _kept(x, s):
    return x if s["ids"] is None else x[:, s["ids"].long()]


def _shape(s, c, z):
    """The definition, in z's type."""
    if c["penal"]:
        prompt, output = (_kept(n, s) for n in _counts(s, c))
        rep = s["rep"].to(z.dtype)[:, None]
        z = torch.where(prompt + output > 0, torch.where(z > 0, z / rep, z * rep), z)
        z = torch.where(output > 0, z - s["freq"].to(z.dtype)[:, None] * output, z)
        z = torch.where(output > 0, z - s["pres"].to(z.dtype)[:, None], z)
    if c["biases"]:
        add = torch.zeros(c["rows"], c["V"] + 1, dtype=torch.float64, device=z.device)
        at = torch.where(s["bias_ids"] < 0, c["V"], s["bias_ids"]).long()
        add.scatter_add_(1, at, s["bias_values"].double())
        z = z + _kept(add[:, :-1], s).to(z.dtype)
    if c["mask"]:
        ids = torch.arange(c["V"], device=z.device) if s["ids"] is None else s["ids"].long()
        words = s["mask"][:, torch.div(ids, 32, rounding_mode="floor")]
        z = torch.where((words >> (ids % 32).to(torch.int32)) & 1 == 1, z, -math.inf)
    return z


def _first_largest(z, s):
    """The lowest id with a row's largest z; -1 for a row that allows none."""
    top = z.amax(1, keepdim=True)
    j = (z == top).to(torch.int8).argmax(1)      # (of equal ones the first)
    ids = j if s["ids"] is None else s["ids"].long()[j]
    return torch.where(top[:, 0] == -math.inf, -1, ids).to(torch.int32)


def _plain_shape(s, c):
    z = _shape(s, c, s["logits"].float())
    if not c["draw"]:
        return z.to(DTYPES[c["out"]])
    return z.to(DTYPES[c["out"]]), _first_largest(z, s)


_PLAIN = {"norm": _plain_norm, "grad": _plain_grad, "quantize": _plain_quantize,
          "product": _plain_product, "shape": _plain_shape}


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------
def _nearest8(v):
    """Magnitudes (64 bits, at most 448 and a rounding) to the nearest e4m3 value: between
    multiples of the step of their power of two, at least 2^-9; of two as near the even one."""
    step = _two(torch.clamp(torch.floor(torch.log2(v.clamp(min=2.0 ** -20))), min=-6.0) - 3)
    # (log2 may round up to the next power of two, where the finer step holds below it)
    step = torch.where((v < 8 * step) & (step > 2.0 ** -9), step / 2, step)
    low = torch.floor(v / step)
    rest = v - low * step
    up = (rest * 2 > step) | ((rest * 2 == step) & (low % 2 == 1))
    return ((low + up.double()) * step).clamp(max=448.0)


def _held64(x, block):
    """The values that x's e4m3 blocks stand for, from 64-bit x."""
    R, d = x.shape
    out = torch.empty_like(x)
    for c0 in range(0, d, 128):
        col = x[:, c0:c0 + 128]
        top = col.abs().amax(1)
        if block > 1:
            pad = torch.cat([top, top.new_zeros(-R % block)]).view(-1, block).amax(1)
            top = pad.repeat_interleave(block)[:R]
        scale = (top / 448).float().double().clamp(min=2.0 ** -126)[:, None]
        out[:, c0:c0 + 128] = torch.sign(col) * _nearest8(col.abs() / scale) * scale
    return out


def _table64(s, c, ids):
    """Rows `ids` of the held table in 64 bits, from the bits of the codes."""
    b = s["codes"].view(torch.uint8)[ids].long()
    e, m = (b >> 3) & 15, (b & 7).double()
    v = torch.where(e > 0, (1 + m / 8) * _two(e - 7), m / 8 * 2.0 ** -6)
    v = torch.where(b >= 128, -v, v)
    f = s["scales"].double()[ids // c["block"]]
    for k in range(f.shape[1]):
        v[:, 128 * k:128 * k + 128] *= f[:, k:k + 1]
    return v


def _exact_norm(s, c):
    x, w = s["x"].double(), s["weight"].double()
    m = x.sum(1, keepdim=True) / c["d"] if c["centre"] else torch.zeros_like(x[:, :1])
    r = ((x - m).pow(2).sum(1, keepdim=True) / c["d"] + EPS).pow(-0.5)
    y = (x - m) * r * w
    return y if s["bias"] is None else y + s["bias"].double()


def _exact_grad(s, c):
    d, w = c["d"], s["weight"].double()
    dx = torch.empty(c["rows"], d, dtype=torch.float64, device=w.device)
    dw, db = torch.zeros_like(w), torch.zeros_like(w)
    step = max(1, (1 << 25) // d)
    for a in range(0, c["rows"], step):
        at = slice(a, a + step)
        dy, r = s["d_out"][at].double(), s["rstd"][at].double()[:, None]
        n = s["x"][at].double()
        if c["centre"]:
            n = n - s["mean"][at].double()[:, None]
        n = n * r
        g = dy * w
        part = n * ((g * n).sum(1, keepdim=True) / d)
        if c["centre"]:
            part = part + g.sum(1, keepdim=True) / d
        dx[at] = r * (g - part)
        dw += (dy * n).sum(0)
        db += dy.sum(0)
    return dx, dw, db if c["bias"] else None


def _exact_shape(s, c):
    """Row by row, from each row's own tokens."""
    y = torch.empty(c["rows"], c["n"], dtype=torch.float64, device=s["logits"].device)
    ids = torch.arange(c["V"], device=y.device) if s["ids"] is None else s["ids"].long()
    for r in range(c["rows"]):
        z = torch.full((c["V"],), -math.inf, dtype=torch.float64, device=y.device)
        z[ids] = s["logits"][r].double()
        if c["penal"]:
            line = s["tokens"][r, :int(s["lengths"][r])].long()
            seen = torch.unique(line)
            rho = float(s["rep"][r])
            z[seen] = torch.where(z[seen] > 0, z[seen] / rho, z[seen] * rho)
            said, times = torch.unique(line[int(s["prompts"][r]):], return_counts=True)
            z[said] -= float(s["freq"][r]) * times + float(s["pres"][r])
        if c["biases"]:
            there = s["bias_ids"][r] >= 0
            z.index_add_(0, s["bias_ids"][r][there].long(), s["bias_values"][r][there].double())
        z = z[ids]
        if c["mask"]:
            bits = (s["mask"][r].long()[:, None] >> torch.arange(32, device=y.device)) % 2
            z = z.masked_fill(bits.reshape(-1)[ids] == 0, -math.inf)
        y[r] = z
    if not c["draw"]:
        return y
    top, j = y.max(1)
    first = torch.where(y == top[:, None], torch.arange(c["n"], device=y.device), c["n"]).amin(1)
    token = ids[torch.where(top > -math.inf, first, j)]
    return y, torch.where(top > -math.inf, token, -1).to(torch.int32)


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["kind"] == "norm":
        return _exact_norm(s, c)
    if c["kind"] == "grad":
        return _exact_grad(s, c)
    if c["kind"] == "shape":
        return _exact_shape(s, c)
    if c["kind"] == "quantize":
        step = max(1, (1 << 25) // c["d"] // 128) * 128
        return torch.cat([_held64(s["x"][a:a + step].double(), c["block"])
                          for a in range(0, c["rows"], step)])
    x = _held64(s["h"].double(), 1)
    ids = torch.arange(c["V"], device=x.device) if s["ids"] is None else s["ids"].long()
    y = torch.empty(c["rows"], c["n"], dtype=torch.float64, device=x.device)
    step = max(1, (1 << 26) // c["d"])
    for a in range(0, c["n"], step):
        y[:, a:a + step] = x @ _table64(s, c, ids[a:a + step]).T
    return y if s["bias"] is None else y + s["bias"][ids].double()
