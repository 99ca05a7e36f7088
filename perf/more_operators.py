"""What the performance of the linear layers in 8-bit integers is measured on: rows quantised, a residual added and normalised into 8 bits,
products of 8-bit rows with 8-bit weights, and a feed-forward layer made of them.

Kinds of case, with the entry points of `paper_2604_15750_amd.api` they go through:
  norm    `dlm_add_norm_q8`: h = residual + x, RMSNorm of h, codes and a scale per row
  rows    `dlm_q8_rows`: codes and a scale per row
  linear  `dlm_q8_gemm` of given codes with a `Q8Weight` (a scale per output channel)
  gated   the same with a gated weight: SwiGLU of the gate and up channels in the product's epilogue
  ffn     the four in turn, as a layer runs them: norm, gated product, rows, product

Where `own` is false the same is computed from elementary torch operations in 32 bits; a code is a quotient rounded next to a border, which takes 64.

Codes are returned as the whole numbers that they stand for, beside their scales: the definition fixes them exactly (a code is 127 t / max|t| rounded to
the nearest, ties to even; the norm's own factor cancels in it), so they have to be equal.

Activations are normal with a few strong channels and rows of different size, residuals the larger part of a sum, gains near 1, weights
normal and quantised by channel.  A gated weight has the gate's channels first, then the up channels.
"""
import math

import torch

own = False  # True: the framework's operators instead of the plain form

EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# (outputs, inputs) of the matrices of the two benchmarked models: QKV, O, down, and the gate and up channels together
MATRICES = {"linear": [(12288, 4096), (4096, 4096), (4096, 12288), (4608, 3584), (3584, 3584), (3584, 18944), (126464, 4096)],
            "gated": [(24576, 4096), (37888, 3584)]}
LAYERS = [(4096, 12288), (3584, 18944), (128, 384)]  # d_model, d_ffn


def listed():
    return [
        # in front of a layer of an in-block pass: a block of the smallest length, the residual stream in fp32; all launch latency
        dict(name="norm_block", kind="norm", rows=8, width=4096, dtype="bf16", residual="f32"),
        # an odd width in fp32
        dict(name="norm_odd", kind="norm", rows=333, width=5003, dtype="f32", residual="f32"),
        # 16 packed prompts of 128, everything in bf16
        dict(name="norm_wide", kind="norm", rows=2048, width=3584, dtype="bf16", residual="bf16"),
        # the input of a down projection for a block: few long rows
        dict(name="rows_block", kind="rows", rows=8, width=18944, dtype="bf16"),
        # ... for a prefill
        dict(name="rows_wide", kind="rows", rows=1500, width=12288, dtype="bf16"),
        # the QKV product of an in-block pass: the weight's bytes
        dict(name="linear_block", kind="linear", rows=8, n=12288, k=4096, out="bf16"),
        # odd in every size, fp32 out
        dict(name="linear_odd", kind="linear", rows=37, n=4999, k=1003, out="f32"),
        # the down projection of 16 sequences inside their blocks: a long sum and few columns
        dict(name="linear_batch", kind="linear", rows=486, n=4096, k=12288, out="bf16"),
        # the QKV product of 16 sequences at a block boundary: the matrix cores' case
        dict(name="linear_wide", kind="linear", rows=2822, n=12288, k=4096, out="bf16"),
        # gate and up of an in-block pass
        dict(name="gated_block", kind="gated", rows=8, n=24576, k=4096, out="bf16"),
        # gate and up of 16 packed prompts of 128: the largest
        dict(name="gated_wide", kind="gated", rows=2048, n=37888, k=3584, out="bf16"),
        # a whole feed-forward layer at a block boundary
        dict(name="ffn_boundary", kind="ffn", rows=152, d=3584, f=18944, dtype="bf16", residual="f32"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(("norm", "rows", "linear", "linear", "gated", "gated", "ffn"))
    c = dict(kind=kind, rows=_log_int(rng, 1, 2822))
    if kind in ("norm", "rows"):
        c.update(width=rng.choice((4096, 3584, 12288, 18944, 128, _log_int(rng, 1, 40000), _log_int(rng, 500, 20000))), dtype=rng.choice(("bf16", "f32")))
        if kind == "norm":
            c["residual"] = "f32" if c["dtype"] == "f32" else rng.choice(("bf16", "f32", "none"))
        while c["rows"] * c["width"] > 2048 * 12288:
            c["rows"] //= 2
        return c
    if kind == "ffn":
        c["d"], c["f"] = rng.choice(LAYERS + [(_log_int(rng, 64, 4096), _log_int(rng, 64, 12288))])
        c.update(dtype="bf16", residual=rng.choice(("bf16", "f32")))
    else:
        c["n"], c["k"] = rng.choice(MATRICES[kind] + [(_log_int(rng, 1, 40000), _log_int(rng, 1, 16000)) for _ in range(3)])
        while c["n"] * c["k"] > 126464 * 4096:
            c["n"] = (c["n"] + 1) // 2
        if kind == "gated":
            c["n"] += c["n"] % 2
        c["out"] = rng.choice(("bf16", "bf16", "f32"))
    while work(c)["flops"] > 5e11:
        c["rows"] //= 2
    return c


# ---- sizes -------------------------------------------------------------------------------------------------------------------

def _bytes(t):
    return {"f32": 4, "bf16": 2, "none": 0}[t]


def _product(rows, n, k, gated, out):
    return dict(bytes=n * k + 4 * n + rows * (k + 4) + rows * (n // 2 if gated else n) * out, flops=2 * rows * n * k)


def work(c):
    rows = c["rows"]
    if c["kind"] == "rows":
        return dict(bytes=rows * (c["width"] * (_bytes(c["dtype"]) + 1) + 4), flops=0)
    if c["kind"] in ("linear", "gated"):
        return _product(rows, c["n"], c["k"], c["kind"] == "gated", _bytes(c["out"]))
    width, x, r = (c["d"] if c["kind"] == "ffn" else c["width"]), _bytes(c["dtype"]), _bytes(c["residual"])
    norm = rows * width * (x + 2 * r) + (2 if c["dtype"] == "bf16" else 4) * width
    if c["kind"] == "norm":
        return dict(bytes=norm + rows * (width + 4), flops=0)
    up, down = _product(rows, 2 * c["f"], width, True, 0), _product(rows, width, c["f"], False, 2)  # what passes between the four is not counted
    weights = 3 * width * c["f"]
    return dict(bytes=norm + weights + 2 * rows * width, flops=up["flops"] + down["flops"])


# ---- inputs, from the seed alone ---------------------------------------------------------------------------------------------

def _normal(seed, stream, shape, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed((seed * 1000003 + stream * 7919 + 31) % (1 << 62))
    return torch.randn(shape, generator=g, device="cuda") * scale


def _padded(rows, width, dtype):
    """New rows whose stride is a multiple of 16 bytes."""
    step = 16 // torch.empty((), dtype=dtype).element_size()
    return torch.zeros((rows, -(-width // step) * step), dtype=dtype, device="cuda")[:, :width]


def _activations(seed, stream, rows, width, dtype, size=1.0):
    strong = 1 + 6 * (_normal(seed, stream + 1, (width,)).abs() > 2.5).float()
    x = _padded(rows, width, TYPES[dtype])
    x.copy_(_normal(seed, stream, (rows, width), size) * strong * torch.exp(0.5 * _normal(seed, stream + 2, (rows, 1))))
    return x


def _norm_inputs(seed, rows, width, dtype, residual):
    x = _activations(seed, 10, rows, width, dtype)
    r = None if residual == "none" else _activations(seed, 20, rows, width, residual, 3.0)
    return x, r, (1 + 0.2 * _normal(seed, 30, (width,))).to(TYPES[dtype])


def _coded(x):
    """Codes (rows padded to 16 bytes) and scales of rows that a program has quantised already."""
    top = x.abs().amax(1, keepdim=True).clamp(min=1e-30)
    codes = _padded(*x.shape, torch.int8)
    codes.copy_(torch.round(x * (127 / top)))
    return codes, (top / 127).reshape(-1)


def _weight_inputs(seed, stream, n, k):
    return _coded(_normal(seed, stream, (n, k), 0.02) * torch.exp(0.3 * _normal(seed, stream + 1, (n, 1))))


def _product_inputs(c, seed):
    return _coded(_activations(seed, 40, c["rows"], c["k"], "f32", 1.5)), _weight_inputs(seed, 50, c["n"], c["k"])


# ---- prepare / run -----------------------------------------------------------------------------------------------------------

def _weight(codes, scale, gated):
    if not own:
        return codes, scale
    from paper_2604_15750_amd import api

    return api.Q8Weight(codes, scale, gated=gated)


def prepare(c, seed):
    rows, s = c["rows"], dict(c=c)
    if c["kind"] in ("norm", "rows"):
        if c["kind"] == "norm":
            s["x"], s["residual"], s["gain"] = _norm_inputs(seed, rows, c["width"], c["dtype"], c["residual"])
            s["h"] = None if s["residual"] is None else _padded(rows, c["width"], s["residual"].dtype)
        else:
            s["x"] = _activations(seed, 10, rows, c["width"], c["dtype"])
        s["codes"], s["scale"] = _padded(rows, c["width"], torch.int8), torch.empty(rows, device="cuda")
        return s
    if c["kind"] == "ffn":
        s["x"], s["residual"], s["gain"] = _norm_inputs(seed, rows, c["d"], c["dtype"], c["residual"])
        s["h"] = _padded(rows, c["d"], s["residual"].dtype)
        s["up"], s["down"] = _weight(*_weight_inputs(seed, 60, 2 * c["f"], c["d"]), True), _weight(*_weight_inputs(seed, 70, c["d"], c["f"]), False)
        for i, width in enumerate((c["d"], c["f"])):
            s["codes%d" % i], s["scale%d" % i] = _padded(rows, width, torch.int8), torch.empty(rows, device="cuda")
        s["act"], s["out"] = _padded(rows, c["f"], torch.bfloat16), _padded(rows, c["d"], torch.bfloat16)
        if own:
            s["ws"] = [s["up"].workspace(rows), s["down"].workspace(rows)]
        return s
    (s["codes"], s["scale"]), w = _product_inputs(c, seed)
    s["w"] = _weight(*w, c["kind"] == "gated")
    s["out"] = _padded(rows, c["n"] // 2 if c["kind"] == "gated" else c["n"], TYPES[c["out"]])
    if own:
        s["ws"] = s["w"].workspace(rows)
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2604_15750_amd import api

    kind = s["c"]["kind"]
    if kind == "rows":
        return api.dlm_q8_rows(s["x"], codes=s["codes"], scale=s["scale"])
    if kind == "norm":
        codes, scale, h = api.dlm_add_norm_q8(s["x"], s["gain"], residual=s["residual"], h=s["h"], eps=EPS, codes=s["codes"], scale=s["scale"])
        return (codes, scale, h) if s["residual"] is not None else (codes, scale)
    if kind != "ffn":
        return api.dlm_q8_gemm(s["w"], s["codes"], s["scale"], out=s["out"], workspace=s["ws"])
    api.dlm_add_norm_q8(s["x"], s["gain"], residual=s["residual"], h=s["h"], eps=EPS, codes=s["codes0"], scale=s["scale0"])
    api.dlm_q8_gemm(s["up"], s["codes0"], s["scale0"], out=s["act"], workspace=s["ws"][0])
    api.dlm_q8_rows(s["act"], codes=s["codes1"], scale=s["scale1"])
    return s["h"], api.dlm_q8_gemm(s["down"], s["codes1"], s["scale1"], out=s["out"], workspace=s["ws"][1])


def _quantise(t):
    """Codes and the largest magnitude of fp32 rows: the quotient in 64 bits, as a code's border may be hit exactly."""
    top = t.abs().amax(1, keepdim=True)
    return torch.where(top > 0, torch.round(127 * t.double() / top.double()), 0.0).to(torch.int8), top.reshape(-1)


def _norm_plain(x, gain, residual):
    h = x if residual is None else (residual.float() + x.float()).to(residual.dtype)
    f = h.float()
    codes, top = _quantise(f * gain.float())
    return codes, top * torch.rsqrt((f * f).mean(1) + EPS) / 127, h


def _product_plain(codes, scale, w, gated, dtype):
    y = torch.matmul(codes.float(), w[0].float().t()) * scale[:, None] * w[1]
    if gated:
        g, u = y.chunk(2, 1)
        y = g / (1 + torch.exp(-g)) * u
    return y.to(dtype)


def _run_plain(s):
    kind = s["c"]["kind"]
    if kind == "rows":
        codes, top = _quantise(s["x"].float())
        return codes, top / 127
    if kind == "norm":
        codes, scale, h = _norm_plain(s["x"], s["gain"], s["residual"])
        return (codes, scale, h) if s["residual"] is not None else (codes, scale)
    if kind != "ffn":
        return _product_plain(s["codes"], s["scale"], s["w"], kind == "gated", s["out"].dtype)
    codes, scale, h = _norm_plain(s["x"], s["gain"], s["residual"])
    codes, top = _quantise(_product_plain(codes, scale, s["up"], True, torch.bfloat16).float())
    return h, _product_plain(codes, top / 127, s["down"], False, torch.bfloat16)


# ---- the same in 64 bits, from the definitions ---------------------------------------------------------------------------------

def _codes64(t):
    """t holds values of 32 bits or fewer."""
    step = t.abs().max(1, keepdim=True).values / 127
    return torch.where(step > 0, t / step, torch.zeros_like(t)), step[:, 0]


def _norm64(x, gain, residual):
    h = x.double()
    if residual is not None:
        h = (residual.double() + h).to(residual.dtype).double()  # h is what the stream holds
    t = (h * gain.double()).float().double()  # ... and its product with the gain a number of 32 bits
    q, step = _codes64(t)
    return torch.round(q), step / (h.pow(2).sum(1) / h.shape[1] + EPS).sqrt(), h


def _product64(codes, scale, w, gated):
    part, step = [], max(1, (1 << 27) // w[0].shape[1])  # channels at a time: the weight in 64 bits is large
    for lo in range(0, w[0].shape[0], step):
        part.append((codes.double() @ w[0][lo:lo + step].double().t().contiguous()) * w[1][lo:lo + step].double())
    y = torch.cat(part, 1) * scale.double().reshape(-1, 1)
    if gated:
        f = y.shape[1] // 2
        y = y[:, :f] * torch.sigmoid(y[:, :f]) * y[:, f:]
    return y


def exact(c, seed):
    rows = c["rows"]
    if c["kind"] == "rows":
        q, step = _codes64(_activations(seed, 10, rows, c["width"], c["dtype"]).double())
        return None, step
    if c["kind"] == "norm":
        x, residual, gain = _norm_inputs(seed, rows, c["width"], c["dtype"], c["residual"])
        q, step, h = _norm64(x, gain, residual)
        return (None, step, h) if residual is not None else (None, step)
    if c["kind"] != "ffn":
        (codes, scale), w = _product_inputs(c, seed)
        return _product64(codes, scale, w, c["kind"] == "gated")
    x, residual, gain = _norm_inputs(seed, rows, c["d"], c["dtype"], c["residual"])
    q, step, h = _norm64(x, gain, residual)
    act = _product64(q, step, _weight_inputs(seed, 60, 2 * c["f"], c["d"]), True).to(torch.bfloat16).double()
    q, step = _codes64(act)
    return h, _product64(torch.round(q), step, _weight_inputs(seed, 70, c["d"], c["f"]), False)
