"""What the performance of the 8-bit KV cache's operators is measured on: queries and keys normalised and rotated, the cache written
and read back, and the attention of packed rows over it.

Kinds of case, with the entry points of `paper_2604_15750_amd.api` they go through:
  rope    `dlm_qk_norm_rope`: RMSNorm of each query and key head and the rotation by the row's position, one pass over the rows of
          a fused QKV product (the V heads behind are left alone)
  write   `dlm_kv8_write` of the spans of packed sequences, and `dlm_kv8_read` of what was written
  read    `dlm_kv8_read` of the cached prefixes of packed sequences
  attend  `dlm_kv8_attention`: packed rows against each sequence's cache, optionally with a mask among the rows (a tree of drafted
          tokens: a row sees the prefix, its ancestors and itself)

Where `own` is false the same is computed from elementary torch operations in 32 bits.

Keys are what a normalised and rotated head holds (unit variance, a common offset, a few strong channels), values are normal with a
spread of magnitudes over the positions, queries lean on the keys' strong channels.
"""
import math

import numpy as np
import torch

own = False  # True: the framework's operators instead of the plain form

# n_q, n_kv, head_dim
HEADS = {"mha": (32, 32, 128), "gqa": (28, 4, 128), "small": (4, 4, 32), "mid": (16, 2, 64)}
THETA, EPS = 10000.0, 1e-5
CODE_MAX = {"e4m3": 448.0, "i8": 127.0}


def listed():
    return [
        # the rows of one in-block pass (a block of the smallest length): all launch latency
        dict(name="rope_block", kind="rope", heads="mha", rows=8, dtype="bf16", first=384),
        # 16 packed prompts of 128: a wide pass, grouped heads
        dict(name="rope_wide", kind="rope", heads="gqa", rows=2048, dtype="bf16", first=0),
        # fp32 rows of a prefill, far positions
        dict(name="rope_f32", kind="rope", heads="mha", rows=600, dtype="f32", first=100000),
        # a committed block, starting inside a block of 32 cached positions
        dict(name="write_block", kind="write", heads="mha", seqs=1, rows=8, first=389, dtype="bf16", format="e4m3"),
        # four ragged prompts, whole blocks of the cache
        dict(name="write_prompts", kind="write", heads="mha", seqs=4, rows=1280, first=0, dtype="bf16", format="i8"),
        # the prefix of one sequence, grouped heads
        dict(name="read_prefix", kind="read", heads="gqa", seqs=1, keys=600, dtype="bf16", format="e4m3"),
        # the prefixes of 16 packed sequences
        dict(name="read_batch", kind="read", heads="mha", seqs=16, keys=768, dtype="bf16", format="i8"),
        # an in-block pass: a block of 8 rows against prompt and decoded blocks
        dict(name="attend_block", kind="attend", heads="mha", seqs=1, rows=8, keys=392, dtype="bf16", format="e4m3", mask=False),
        # a tree of 48 drafted tokens behind 4096 cached positions, grouped heads
        dict(name="attend_tree", kind="attend", heads="gqa", seqs=1, rows=48, keys=4144, dtype="bf16", format="e4m3", mask=True),
        # single tokens of 24 long sequences, grouped heads: the cache's read rate
        dict(name="attend_tokens", kind="attend", heads="gqa", seqs=24, rows=1, keys=8192, dtype="bf16", format="i8", mask=False),
        # a prompt of 1024 with 256 look-ahead positions: the matrix cores' case
        dict(name="attend_prefill", kind="attend", heads="mha", seqs=1, rows=1280, keys=1280, dtype="bf16", format="e4m3", mask=False),
        # fp32 rows of two long blocks late in a generation
        dict(name="attend_f32", kind="attend", heads="mha", seqs=2, rows=37, keys=1537, dtype="f32", format="i8", mask=False),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(("rope", "write", "read") + ("attend",) * 4)
    c = dict(kind=kind, heads=rng.choice(("mha", "gqa", "mha", "gqa", "small", "mid")), dtype=rng.choice(("bf16", "bf16", "f32")))
    if kind == "rope":
        c.update(rows=_log_int(rng, 1, 2048), first=rng.choice((0, rng.randrange(1, 4000), rng.randrange(4000, 1 << 20))))
        return c
    c.update(seqs=_log_int(rng, 1, 24), format=rng.choice(("e4m3", "i8")))
    if kind == "write":
        c.update(rows=min(_log_int(rng, 1, 1280), max(1, 5120 // c["seqs"])), first=rng.choice((0, rng.randrange(1, 2000))))
    elif kind == "read":
        c.update(keys=min(_log_int(rng, 1, 8192), max(1, 12288 // c["seqs"])))
    else:
        c.update(mask=rng.random() < 0.35)
        rows = _log_int(rng, 1, 64) if c["mask"] else rng.choice((1, _log_int(rng, 1, 128), _log_int(rng, 1, 1280)))
        c.update(rows=rows, keys=max(rows, _log_int(rng, 16, 16384)))
        while work(c)["flops"] > 2.6e10 or c["seqs"] * c["keys"] > 24 * 8192:  # no more than the largest listed cases
            if c["seqs"] > 1:
                c["seqs"] = max(1, c["seqs"] // 2)
            elif c["keys"] > c["rows"]:
                c["keys"] = max(c["rows"], c["keys"] // 2)
            else:
                c["rows"] //= 2
    return c


# ---- sizes -------------------------------------------------------------------------------------------------------------------

def _ragged(n, b):
    """Length of sequence b where the longest is n: the first has n, the others between half of it and all of it."""
    return max(1, n - (n // 2) * ((5 * b) % 8) // 7)


def _spans(c):
    """Per sequence (rows of the call, first cached position they have, cached positions in all)."""
    out = []
    for b in range(c["seqs"]):
        if c["kind"] == "write":
            n, first = _ragged(c["rows"], b), c["first"] + 3 * b
            out.append((n, first, first + n))
        elif c["kind"] == "read":
            n = _ragged(c["keys"], b)
            out.append((n, 0, n))
        else:
            n = _ragged(c["rows"], b)
            keys = max(n, _ragged(c["keys"], b))
            out.append((n, keys - n, keys))
    return out


def _offsets(spans):
    off = [0]
    for n, _, _ in spans:
        off.append(off[-1] + n)
    return off


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def work(c):
    n_q, n_kv, hd = HEADS[c["heads"]]
    es = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "rope":
        n = c["rows"] * (n_q + n_kv) * hd
        return dict(bytes=2 * n * es + 4 * c["rows"] + 2 * hd * es, flops=8 * n)
    spans = _spans(c)
    rows, keys = sum(s[0] for s in spans), sum(s[2] for s in spans)
    vector = n_kv * (2 * hd + 2)  # K and V of a cached position: codes and two scales
    if c["kind"] == "write":  # rows read and codes written, codes read and values written
        return dict(bytes=2 * rows * (vector + 2 * n_kv * hd * es), flops=0)
    if c["kind"] == "read":
        return dict(bytes=rows * (vector + 2 * n_kv * hd * es), flops=0)
    return dict(bytes=keys * vector + 2 * rows * n_q * hd * es + (rows * 4 * _words(c) if c["mask"] else 0),
                flops=sum(4 * n * k for n, _, k in spans) * n_q * hd)


def _words(c):
    return (c["rows"] + 31) // 32


# ---- inputs, from the seed alone ---------------------------------------------------------------------------------------------

def _normal(seed, stream, shape, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed((seed * 1000003 + stream * 7919 + 31) % (1 << 62))
    return torch.randn(shape, generator=g, device="cuda") * scale


def _channels(seed, n_kv, hd):
    """Per key head a common offset and a few strong channels."""
    strong = 1 + 3 * (_normal(seed, 1, (n_kv, hd)).abs() > 2).float()
    return strong, 0.5 * _normal(seed, 2, (n_kv, hd))


def _keys_values(c, seed, n, stream):
    _, n_kv, hd = HEADS[c["heads"]]
    strong, offset = _channels(seed, n_kv, hd)
    k = (_normal(seed, stream, (n, n_kv, hd)) + offset) * strong
    v = _normal(seed, stream + 1, (n, n_kv, hd)) * torch.exp(0.7 * _normal(seed, stream + 2, (n, n_kv, 1)))
    return k.to(_dtype(c)), v.to(_dtype(c))


def _queries(c, seed, rows):
    n_q, n_kv, hd = HEADS[c["heads"]]
    strong, offset = _channels(seed, n_kv, hd)
    q = _normal(seed, 30, (rows, n_kv, n_q // n_kv, hd)) + (0.3 * offset / strong)[None, :, None]
    return q.reshape(rows, n_q, hd).to(_dtype(c))


def _tree(c, seed):
    """Ancestors' bits of random trees, one per sequence: int32 [rows, words], bit j of a row: it sees node j of its sequence."""
    rng, parts = np.random.default_rng(seed * 7 + 1), []
    for n, _, _ in _spans(c):
        see = np.zeros((n, 32 * _words(c)), dtype=bool)
        for i in range(n):
            p = int(rng.integers(max(-1, i - 8), i))
            if p >= 0:
                see[i] = see[p]
            see[i, i] = True
        parts.append(see)
    see = np.concatenate(parts).reshape(-1, _words(c), 32).astype(np.uint64)
    return torch.from_numpy((see << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32).view(np.int32)).cuda()


def _rope_inputs(c, seed):
    n_q, n_kv, hd = HEADS[c["heads"]]
    rows = c["rows"]
    qkv = (_normal(seed, 20, (rows, (n_q + 2 * n_kv) * hd)) * torch.exp(0.5 * _normal(seed, 21, (rows, 1)))).to(_dtype(c))
    gains = [(1 + 0.2 * _normal(seed, 22 + i, (hd,))).to(_dtype(c)) for i in range(2)]
    positions = torch.arange(rows, device="cuda", dtype=torch.int32) % max(1, (rows + 15) // 16 if rows >= 1024 else rows) + c["first"]
    return qkv, gains, positions.to(torch.int32)


# ---- prepare / run -----------------------------------------------------------------------------------------------------------

def prepare(c, seed):
    n_q, n_kv, hd = HEADS[c["heads"]]
    if c["kind"] == "rope":
        qkv, (gq, gk), positions = _rope_inputs(c, seed)
        return dict(c=c, qkv=qkv, gq=gq, gk=gk, positions=positions, out=torch.empty_like(qkv))
    spans = _spans(c)
    off, total = _offsets(spans), max(s[2] for s in spans)
    s = dict(c=c, spans=spans, off=off, starts=[x[1] for x in spans], ends=[x[2] for x in spans])
    if own:
        from paper_2604_15750_amd import api

        s["cache"] = api.Kv8Cache(len(spans), total, n_kv, hd, c["format"], "cuda")
    if c["kind"] == "write":
        s["k"], s["v"] = _keys_values(c, seed, off[-1], 10)
        s["out"] = torch.empty_like(s["k"]), torch.empty_like(s["v"])
        return s
    if not own:
        s["codes"] = [torch.zeros((len(spans), n_kv, total, hd), dtype=torch.int8, device="cuda") for _ in "kv"]
        s["scale"] = [torch.zeros((len(spans), n_kv, total, 1), device="cuda") for _ in "kv"]
    for b, (_, _, n) in enumerate(spans):  # what earlier passes left in the cache
        rows = _keys_values(c, seed, n, 100 + 10 * b)
        if own:
            api.dlm_kv8_write(s["cache"], *rows, [0, n], [0], slot=[b])
        else:
            for i, x in enumerate(rows):
                code, scale = _quantise(x.float(), c["format"])
                s["codes"][i][b, :, :n] = code.view(torch.int8).permute(1, 0, 2)
                s["scale"][i][b, :, :n] = scale.permute(1, 0, 2)
    if c["kind"] == "read":
        s["out"] = tuple(torch.empty((off[-1], n_kv, hd), dtype=_dtype(c), device="cuda") for _ in "kv")
        return s
    s["q"] = _queries(c, seed, off[-1])
    s["mask"] = _tree(c, seed) if c["mask"] else None
    s["out"] = torch.empty_like(s["q"])
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2604_15750_amd import api

    c = s["c"]
    n_q, n_kv, hd = HEADS[c["heads"]]
    if c["kind"] == "rope":
        api.dlm_qk_norm_rope(s["qkv"], s["positions"], n_q, n_kv, hd, s["gq"], s["gk"], EPS, THETA, out=s["out"])
        return s["out"][:, :(n_q + n_kv) * hd]
    if c["kind"] == "attend":
        return api.dlm_kv8_attention(s["cache"], s["q"], s["off"], s["ends"], mask=s["mask"], out=s["out"])
    if c["kind"] == "write":
        api.dlm_kv8_write(s["cache"], s["k"], s["v"], s["off"], s["starts"])
    return api.dlm_kv8_read(s["cache"], s["off"], s["starts"], k=s["out"][0], v=s["out"][1])


def _quantise(x, fmt):
    """Codes and scales of vectors x [..., hd] in 32 bits: the scale is the smallest power of two 2^E, E in [-60, 60], for which the
    largest magnitude has a code."""
    frac, e = torch.frexp(x.abs().amax(-1, keepdim=True))
    top = CODE_MAX[fmt]
    bits = 9 if fmt == "e4m3" else 7
    e = (e - bits + (frac > top / 2.0 ** bits)).clamp(-60, 60)
    y = torch.ldexp(x, -e).clamp(-top, top)
    return (y.to(torch.float8_e4m3fn) if fmt == "e4m3" else torch.round(y).to(torch.int8)), torch.ldexp(torch.ones_like(frac), e)


def _values(code, fmt):
    return (code.view(torch.float8_e4m3fn) if fmt == "e4m3" else code).float()


def _run_plain(s):
    c = s["c"]
    n_q, n_kv, hd = HEADS[c["heads"]]
    if c["kind"] == "rope":
        rows = s["qkv"].shape[0]
        x = s["qkv"][:, :(n_q + n_kv) * hd].float().view(rows, n_q + n_kv, hd)
        gain = torch.cat([s["gq"].float().expand(n_q, hd), s["gk"].float().expand(n_kv, hd)])
        y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain
        freq = THETA ** (-2.0 * torch.arange(hd // 2, device="cuda", dtype=torch.float64) / hd)
        ang = s["positions"].double()[:, None, None] * freq  # far positions: the angle needs 64 bits
        cos, sin = ang.cos().float(), ang.sin().float()
        y1, y2 = y[..., :hd // 2], y[..., hd // 2:]
        return torch.cat([y1 * cos - y2 * sin, y2 * cos + y1 * sin], -1).reshape(rows, -1).to(s["qkv"].dtype)
    if c["kind"] == "write":
        out = []
        for x in (s["k"], s["v"]):
            code, scale = _quantise(x.float(), c["format"])
            out.append((code.float() * scale).to(x.dtype))
        return tuple(out)
    if c["kind"] == "read":
        return tuple(torch.cat([(_values(code[b, :, :n], c["format"]) * scale[b, :, :n]).permute(1, 0, 2) for b, (_, _, n) in enumerate(s["spans"])])
                     .to(s["out"][0].dtype) for code, scale in zip(s["codes"], s["scale"]))
    out = []
    for b, (n, first, keys) in enumerate(s["spans"]):
        K, V = (_values(s["codes"][i][b, :, :keys], c["format"]) * s["scale"][i][b, :, :keys] for i in range(2))
        q = s["q"][s["off"][b]:s["off"][b + 1]].float().view(n, n_kv, n_q // n_kv, hd).permute(1, 2, 0, 3).reshape(n_kv, -1, hd).contiguous()
        z = torch.matmul(q, K.transpose(1, 2).contiguous()).view(n_kv, n_q // n_kv, n, keys) / math.sqrt(hd)
        if s["mask"] is not None:
            words = s["mask"][s["off"][b]:s["off"][b + 1]]
            see = ((words[:, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1).view(n, -1)[:, :n] != 0
            z[..., first:] = torch.where(see, z[..., first:], float("-inf"))
        p = torch.exp(z - z.amax(-1, keepdim=True))
        p = (p / p.sum(-1, keepdim=True)).view(n_kv, -1, keys)
        o = torch.matmul(p, V.contiguous()).view(n_kv, n_q // n_kv, n, hd).permute(2, 0, 1, 3)
        out.append(o.reshape(n, n_q, hd))
    return torch.cat(out).to(s["q"].dtype)


# ---- the same in 64 bits, from the definitions ---------------------------------------------------------------------------------

def _stored64(x, fmt):
    """What a vector is held as: the nearest values of the format on the scale of its largest magnitude."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -80) / CODE_MAX[fmt])).clamp(-60, 60)
    e = torch.where(top > CODE_MAX[fmt] * torch.exp2(e), e + 1, e)  # (the logarithm's own rounding next to a power of two)
    e = torch.where(top <= CODE_MAX[fmt] * torch.exp2(e - 1), e - 1, e).clamp(-60, 60)
    y = x / torch.exp2(e)
    if fmt == "i8":
        return torch.round(y) * torch.exp2(e)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)  # three fraction bits, 2^-9 below the normal values
    return torch.round(y / step) * step * torch.exp2(e)


def exact(c, seed):
    n_q, n_kv, hd = HEADS[c["heads"]]
    group = n_q // n_kv
    if c["kind"] == "rope":
        qkv, (gq, gk), positions = _rope_inputs(c, seed)
        out = []
        turn = torch.exp(-math.log(THETA) * torch.arange(0, hd, 2, device="cuda", dtype=torch.float64) / hd)
        w = torch.polar(torch.ones(c["rows"], 1, hd // 2, dtype=torch.float64, device="cuda"), positions.double()[:, None, None] * turn)
        for first, n, gain in ((0, n_q, gq), (n_q, n_kv, gk)):
            x = qkv.double()[:, first * hd:(first + n) * hd].reshape(-1, n, hd)
            x = gain.double() * x / (x.pow(2).sum(-1, keepdim=True) / hd + EPS).sqrt()
            z = torch.complex(x[..., :hd // 2].contiguous(), x[..., hd // 2:].contiguous()) * w
            out.append(torch.cat([z.real, z.imag], -1).reshape(c["rows"], -1))
        return torch.cat(out, 1)
    spans = _spans(c)
    if c["kind"] == "write":
        return tuple(_stored64(x, c["format"]) for x in _keys_values(c, seed, _offsets(spans)[-1], 10))
    stored = [[_stored64(x, c["format"]) for x in _keys_values(c, seed, n, 100 + 10 * b)] for b, (_, _, n) in enumerate(spans)]
    if c["kind"] == "read":
        return tuple(torch.cat([kv[i] for kv in stored]) for i in range(2))
    off = _offsets(spans)
    q, tree = _queries(c, seed, off[-1]).double(), _tree(c, seed).cpu().numpy().view(np.uint32) if c["mask"] else None
    out = torch.empty_like(q)
    for b, (n, first, keys) in enumerate(spans):
        see = torch.ones((n, keys), dtype=torch.bool)
        if tree is not None:
            bits = np.unpackbits(tree[off[b]:off[b + 1]].view(np.uint8), axis=1, bitorder="little")[:, :n]
            see[:, first:] = torch.from_numpy(bits != 0)
        see = see.cuda()
        for h in range(n_q):
            K, V = (x[:, h // group].contiguous() for x in stored[b])
            z = q[off[b]:off[b + 1], h].contiguous() @ K.t().contiguous() * hd ** -0.5
            out[off[b]:off[b + 1], h] = torch.softmax(z.masked_fill(~see, -math.inf), -1) @ V
    return out
