"""Operators of a decoder's feed-forward half on 4-bit weights with group scales: what is measured, in plain form and through
the framework.

The set: uniform 4-bit quantisation of a weight matrix with a scale and a zero point per group of 32, 64 or 128 columns (and its
inverse), products of such a matrix with one or many token vectors, the gated product act(Wg x) * (Wu x) of two such matrices,
and the root-mean-square norm with the residual's addition whose 8-bit rows these products read.

`run` computes the plain form with elementary torch operations in 32 bits; with `own` set it makes the framework's calls.  Both
take the weights in the framework's stored form, so both decode them within the call.
"""
import functools
import math

import torch

own = False

STREAM = {"f16": torch.float16, "bf16": torch.bfloat16}
OUT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# the nibble that holds column e of a word's eight
PLACE = [0, 4, 1, 5, 2, 6, 3, 7]


# ---------------------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # the repository's smallest configuration, finest groups, with the error per row: latency
        {"name": "quantize 256x512 g32", "op": "quantize", "rows": 256, "cols": 512, "group": 32, "importance": False},
        # the benchmark's matrix, importance-weighted error as the clustering reports it
        {"name": "quantize 4096x11008 g128", "op": "quantize", "rows": 4096, "cols": 11008, "group": 128, "importance": True},
        # one decoded token: an attention projection
        {"name": "matvec t1 4096x4096", "op": "matvec", "tokens": 1, "rows": 4096, "cols": 4096, "group": 128, "x": "f16", "out": "f32", "pad": 0},
        # eight requests decoded together: the down projection, activations in 8 bits
        {"name": "matvec t8 4096x11008 8bit", "op": "matvec", "tokens": 8, "rows": 4096, "cols": 11008, "group": 64, "x": "i8", "out": "f16", "pad": 0},
        # ragged in every direction, tokens of a short prompt
        {"name": "matvec t77 1000x3001", "op": "matvec", "tokens": 77, "rows": 1000, "cols": 3001, "group": 32, "x": "f16", "out": "f32", "pad": 7},
        # a prompt of a thousand tokens
        {"name": "matvec t1024 11008x4096", "op": "matvec", "tokens": 1024, "rows": 11008, "cols": 4096, "group": 128, "x": "bf16", "out": "bf16", "pad": 0},
        # one decoded token through gate and up
        {"name": "gated t1 11008x4096", "op": "gated", "tokens": 1, "rows": 11008, "cols": 4096, "group": 128, "x": "f16", "out": "f16", "act": "silu", "pad": 0},
        # a batch of sixteen, activations in 8 bits
        {"name": "gated t16 11008x4096 8bit", "op": "gated", "tokens": 16, "rows": 11008, "cols": 4096, "group": 128, "x": "i8", "out": "bf16", "act": "silu", "pad": 0},
        # a prompt through the wider layer's gate and up
        {"name": "gated t300 22016x8192", "op": "gated", "tokens": 300, "rows": 22016, "cols": 8192, "group": 128, "x": "bf16", "out": "bf16", "act": "gelu", "pad": 0},
        # one token's row, 8-bit output
        {"name": "norm t1 4096 8bit", "op": "norm", "tokens": 1, "cols": 4096, "x": "f16", "eight": True, "pad": 0},
        # a prompt of two thousand tokens in the wider layer
        {"name": "norm t2048 8192", "op": "norm", "tokens": 2048, "cols": 8192, "x": "bf16", "eight": False, "pad": 0},
        # the half layer of four decoded tokens: norm to 8 bits, gate and up, down
        {"name": "feed forward t4 4096 11008", "op": "ffn", "tokens": 4, "cols": 4096, "hidden": 11008, "group": 128, "x": "f16", "act": "silu", "pad": 0},
    ]


MOST_PRODUCTS = 300 * 22016 * 8192 * 2


def draw(rng):
    def size(low, high):
        n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
        kind = rng.random()
        if kind < 0.5:
            n = max(low, n // 64 * 64)
        elif kind < 0.7:
            n = n | 1
        return min(n, high)

    op = rng.choice(["quantize", "matvec", "matvec", "gated", "gated", "norm", "ffn"])
    group = rng.choice([32, 64, 128])
    pad = rng.choice([0, 0, 8, 3])
    if op == "quantize":
        return {"op": op, "rows": size(64, 8192), "cols": size(64, 11008), "group": group, "importance": rng.random() < 0.5}
    if op == "norm":
        x = rng.choice(["f16", "bf16"])
        return {"op": op, "tokens": size(1, 2048), "cols": size(64, 8192), "x": x, "eight": rng.random() < 0.5, "pad": pad}
    if op == "ffn":
        cols, hidden = size(128, 8192), size(128, 11008)
        tokens = min(size(1, 64), max(1, MOST_PRODUCTS // (3 * cols * hidden)))
        return {"op": op, "tokens": tokens, "cols": cols, "hidden": hidden, "group": group, "x": rng.choice(["f16", "bf16"]), "act": rng.choice(["silu", "gelu"]), "pad": pad}
    rows, cols = size(64, 11008), size(64, 11008)
    tokens = min(size(1, 1024), max(1, MOST_PRODUCTS // (rows * cols * 2)))
    case = {"op": op, "tokens": tokens, "rows": rows, "cols": cols, "group": group, "x": rng.choice(["f16", "bf16", "i8"]), "out": rng.choice(["f32", "f16", "bf16"]), "pad": pad}
    if op == "gated":
        case["act"] = rng.choice(["silu", "gelu"])
    return case


def stored_bytes(rows, cols, group):
    """What a matrix needs at least: half a byte a weight, a 16-bit scale and a 4-bit zero point a group."""
    return rows * cols / 2 + rows * -(-cols // group) * 2.5


def work(case):
    op = case["op"]
    if op == "quantize":
        n = case["rows"] * case["cols"]
        held = stored_bytes(case["rows"], case["cols"], case["group"])
        # weights and importances in, the stored form out and in again, binary16 values and errors out
        return {"bytes": n * (2 + (4 if case["importance"] else 0)) + 2 * held + n * 2 + case["rows"] * 4, "flops": 8 * n}
    if op == "norm":
        n, rows = case["tokens"] * case["cols"], case["tokens"]
        return {"bytes": n * (2 + 2 + 2 + (1 if case["eight"] else 2)) + case["cols"] * 2 + (rows * 4 if case["eight"] else 0), "flops": 6 * n}
    if op == "ffn":
        t, c, h = case["tokens"], case["cols"], case["hidden"]
        held = 2 * stored_bytes(h, c, case["group"]) + stored_bytes(c, h, case["group"])
        return {"bytes": held + t * c * (2 + 2 + 2 + 2) + c * 2, "flops": 6 * t * c * h}
    t, r, c = case["tokens"], case["rows"], case["cols"]
    mats = 2 if op == "gated" else 1
    x = t * c + t * 4 if case["x"] == "i8" else t * c * 2
    y = t * r * (4 if case["out"] == "f32" else 2)
    return {"bytes": mats * stored_bytes(r, c, case["group"]) + x + y, "flops": 2 * mats * t * r * c}


# ---------------------------------------------------------------------------------------------------------------- plain form

def group_quantize(w, group):
    """Codes (0..15), scales (binary16) and zero points per group of columns; w binary32 [rows, cols]."""
    rows, cols = w.shape
    groups = -(-cols // group)
    v = torch.zeros((rows, groups * group), dtype=torch.float32, device=w.device)
    v[:, :cols] = w
    v = v.view(rows, groups, group)
    low = v.amin(dim=2).clamp(max=0.0)
    high = v.amax(dim=2).clamp(min=0.0)
    scale = ((high - low) / 15.0).half()
    s = scale.float()
    some = s > 0
    by = torch.where(some, s, torch.ones_like(s))
    zero = torch.where(some, torch.round(-low / by).clamp(0, 15), torch.zeros_like(s))
    codes = (torch.round(v / by[:, :, None]) + zero[:, :, None]).clamp(0, 15) * some[:, :, None]
    return codes.view(rows, groups * group)[:, :cols].to(torch.int32), scale, zero.to(torch.int32)


def store(codes, scale, zero, group):
    """The stored form: records of 16 rows x 128 columns, one row of records after another.  A record holds, for each of its rows, 16
    words of codes -- word 4 p + t has columns 32 t + 8 p to 32 t + 8 p + 7 of the record, column e of them in nibble PLACE[e] --
    and behind the 256 words one word for every row and group: the scale's bits, the zero point above them."""
    rows, cols = codes.shape
    rt, ct, per = -(-rows // 16), -(-cols // 128), 128 // group
    c = torch.zeros((rt * 16, ct * 128), dtype=torch.int64, device=codes.device)
    c[:rows, :cols] = codes
    c = c.view(rt, 16, ct, 4, 4, 8)                                      # row, t, p, e
    shift = torch.tensor([4 * p for p in PLACE], dtype=torch.int64, device=codes.device)
    words = (c << shift).sum(dim=-1).permute(0, 2, 1, 4, 3)              # rt, ct, row, p, t
    m = torch.zeros((rt * 16, ct * per), dtype=torch.int64, device=codes.device)
    m[:rows, :scale.shape[1]] = (scale.view(torch.int16).to(torch.int64) & 0xffff) | (zero.to(torch.int64) << 16)
    m = m.view(rt, 16, ct, per).permute(0, 2, 1, 3)
    both = torch.cat([words.reshape(rt, ct, 256), m.reshape(rt, ct, 16 * per)], dim=2)
    both = torch.where(both >= 2 ** 31, both - 2 ** 32, both).to(torch.int32)
    return both.contiguous().view(-1).view(torch.uint8)


def weights_of(q):
    """The binary32 matrix that a stored form stands for."""
    rows, cols, group = q["rows"], q["cols"], q["group"]
    rt, ct, per = -(-rows // 16), -(-cols // 128), 128 // group
    both = q["tiles"].view(torch.int32).view(rt, ct, 256 + 16 * per)
    words = both[:, :, :256].view(rt, ct, 16, 4, 4)                      # row, p, t
    shift = torch.tensor([4 * p for p in PLACE], dtype=torch.int32, device=words.device)
    codes = (words[..., None] >> shift) & 15                             # row, p, t, e
    codes = codes.permute(0, 2, 1, 4, 3, 5).reshape(rt * 16, ct * 128)
    m = both[:, :, 256:].view(rt, ct, 16, per).permute(0, 2, 1, 3).reshape(rt * 16, ct * per)
    scale = (m & 0xffff).to(torch.int16).view(torch.float16).float()
    zero = m >> 16
    w = (codes.view(rt * 16, ct * per, group) - zero[:, :, None]).float() * scale[:, :, None]
    return w.view(rt * 16, ct * 128)[:rows, :cols]


def activation(name, g):
    if name == "silu":
        return g / (1.0 + torch.exp(-g))
    return 0.5 * g * (1.0 + torch.tanh(0.7978845608028654 * (g + 0.044715 * g * g * g)))


def plain_rows(s):
    x = s["x"].float()
    return x * s["x_scale"][:, None] if s["x_scale"] is not None else x


def plain_norm(x, residual, weight, eps, eight):
    """(the new residual stream, the normalised rows in binary32, or their 8-bit codes as numbers and the scales)"""
    h = x.float() + residual.float()
    rstd = 1.0 / torch.sqrt((h * h).mean(dim=1) + eps)
    p = h * weight.float()
    if not eight:
        return h.to(x.dtype), p * rstd[:, None], None
    a = p.abs().amax(dim=1)
    by = torch.where(a > 0, a, torch.ones_like(a)).double()
    codes = torch.round(p.double() * 127.0 / by[:, None]).float()
    return h.to(x.dtype), codes, a * rstd / 127.0


def plain_run(s):
    c = s["case"]
    if c["op"] == "quantize":
        w = s["W"].float()
        codes, scale, zero = group_quantize(w, c["group"])
        width = torch.arange(c["cols"], device=w.device) // c["group"]
        value = (codes - zero[:, width]).float() * scale.float()[:, width]
        d = w - value
        e = d * d
        return value.half(), (e if s["G"] is None else e * s["G"]).sum(dim=1)
    if c["op"] == "matvec":
        return (plain_rows(s) @ weights_of(s["q"]).t()).to(OUT[c["out"]])
    if c["op"] == "gated":
        x = plain_rows(s)
        return (activation(c["act"], x @ weights_of(s["gate"]).t()) * (x @ weights_of(s["up"]).t())).to(OUT[c["out"]])
    if c["op"] == "norm":
        stream, rows, scale = plain_norm(s["x"], s["residual"], s["weight"], s["eps"], c["eight"])
        return (stream, rows * scale[:, None]) if c["eight"] else (stream, rows.to(s["x"].dtype))
    stream, rows, scale = plain_norm(s["x"], s["residual"], s["weight"], s["eps"], True)
    x = rows * scale[:, None]
    hidden = activation(c["act"], x @ weights_of(s["gate"]).t()) * (x @ weights_of(s["up"]).t())
    return stream, (hidden.to(s["x"].dtype).float() @ weights_of(s["down"]).t()).to(s["x"].dtype)


# ---------------------------------------------------------------------------------------------------------------- the framework

@functools.cache
def context():
    """The handle that a program makes once: the device's default stream, the smallest workspace (its status word)."""
    from paper_2412_04180_b200.skim import Skim
    ctx = Skim(device=torch.cuda.current_device())
    ctx.set_workspace(torch.empty(4096, dtype=torch.uint8, device="cuda"))
    return ctx


def own_run(s):
    c, ctx = s["case"], context()
    if c["op"] == "quantize":
        q = ctx.grouped_quantize(s["W"], c["group"], importance=s["G"], want_err=True)
        return ctx.grouped_dequantize(q), q["err"]
    if c["op"] == "matvec":
        return ctx.grouped_matvec(s["q"], s["x"], x_scale=s["x_scale"], out_dtype=OUT[c["out"]])
    if c["op"] == "gated":
        return ctx.grouped_gated(s["gate"], s["up"], s["x"], x_scale=s["x_scale"], activation=c["act"], out_dtype=OUT[c["out"]])
    if c["op"] == "norm":
        out, scale, stream = ctx.add_rmsnorm(s["x"], s["weight"], eps=s["eps"], residual=s["residual"], out_dtype=torch.int8 if c["eight"] else None)
        return (stream, out * scale[:, None]) if c["eight"] else (stream, out)
    out, stream = ctx.feed_forward(s["x"], s["weight"], s["gate"], s["up"], s["down"], eps=s["eps"], residual=s["residual"], activation=c["act"], eight_bit=True)
    return stream, out


def run(s):
    return own_run(s) if own else plain_run(s)


# ---------------------------------------------------------------------------------------------------------------- inputs

def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda")

    def matrix(rows, cols):
        """Bell-shaped weights of standard deviation 0.02, one in a thousand ten times as far out."""
        w = normal(rows, cols) * 0.02
        far = torch.rand((rows, cols), generator=gen, device="cuda") < 1e-3
        return torch.where(far, w * 10.0, w).half()

    def held(rows, cols):
        codes, scale, zero = group_quantize(matrix(rows, cols).float(), case["group"])
        return {"tiles": store(codes, scale, zero, case["group"]), "rows": rows, "cols": cols, "group": case["group"]}

    def padded(v):
        """The same rows, a few unused values between them where the case says so."""
        room = torch.zeros((v.shape[0], v.shape[1] + case["pad"]), dtype=v.dtype, device=v.device)
        room[:, :v.shape[1]] = v
        return room[:, :v.shape[1]]

    def channels(cols):
        """Channels of different strength, a few of them eight times as strong."""
        c = torch.exp(0.3 * normal(cols))
        c[torch.randint(cols, (max(1, cols // 1000),), generator=gen, device="cuda")] *= 8.0
        return c

    s = {"case": dict(case)}
    op = case["op"]
    if op == "quantize":
        s["W"] = matrix(case["rows"], case["cols"])
        s["G"] = torch.exp(1.5 * normal(case["rows"], case["cols"])) if case["importance"] else None
        return s
    if op in ("norm", "ffn"):
        t, cols, dtype = case["tokens"], case["cols"], STREAM[case["x"]]
        s["x"] = padded((normal(t, cols) * 0.5).to(dtype))
        s["residual"] = padded((normal(t, cols) * 2.0 * channels(cols)).to(dtype))
        s["weight"] = (1.0 + 0.2 * normal(cols)).to(dtype)
        s["eps"] = 1e-5
        if op == "ffn":
            s["gate"], s["up"], s["down"] = held(case["hidden"], cols), held(case["hidden"], cols), held(cols, case["hidden"])
        return s
    x = normal(case["tokens"], case["cols"]) * channels(case["cols"])
    s["x_scale"] = None
    if case["x"] == "i8":
        s["x_scale"] = x.abs().amax(dim=1) / 127.0
        s["x"] = padded(torch.round(x / s["x_scale"][:, None]).to(torch.int8))
    else:
        s["x"] = padded(x.to(STREAM[case["x"]]))
    if op == "matvec":
        s["q"] = held(case["rows"], case["cols"])
    else:
        s["gate"], s["up"] = held(case["rows"], case["cols"]), held(case["rows"], case["cols"])
    return s


# ---------------------------------------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "quantize":
        w = s["W"].double()
        value, err = torch.empty_like(w), torch.zeros(case["rows"], dtype=torch.float64, device=w.device)
        for first in range(0, case["cols"], case["group"]):
            part = w[:, first:first + case["group"]]
            none = torch.zeros((case["rows"], 1), dtype=torch.float64, device=w.device)
            high, low = torch.maximum(part.amax(1, True), none), torch.minimum(part.amin(1, True), none)
            # the definition's roundings of the scale: the difference and the quotient to binary32, then to binary16
            step = ((high - low).float().double() / 15.0).float().half().double()
            div = torch.where(step > 0, step, torch.ones_like(step))
            origin = torch.round(-low / div).clamp(0.0, 15.0)
            there = ((torch.round(part / div) + origin).clamp(0.0, 15.0) - origin) * step
            value[:, first:first + case["group"]] = there
            miss = (part - there) ** 2
            if s["G"] is not None:
                miss = miss * s["G"][:, first:first + case["group"]].double()
            err += miss.sum(1)
        return value, err

    def matrix(q):
        rt, ct, per = -(-q["rows"] // 16), -(-q["cols"] // 128), 128 // q["group"]
        record = q["tiles"].view(rt, ct, 1024 + 64 * per)
        byte = record[:, :, :1024].reshape(rt, ct, 16, 4, 4, 4)          # row, p, t, byte of the word
        out = torch.empty((rt, 16, ct, 4, 4, 8), dtype=torch.float64, device=byte.device)
        place = {p: e for e, p in enumerate(PLACE)}
        for b in range(4):
            for high in range(2):
                nibble = (byte[..., b] >> (4 * high)) & 15
                out[..., place[2 * b + high]] = nibble.permute(0, 2, 1, 4, 3).double()
        tail = record[:, :, 1024:].reshape(rt, ct, 16, per, 4)
        scale = tail[..., :2].contiguous().view(torch.float16)[..., 0].double()
        origin = tail[..., 2].double()
        out = out.view(rt, 16, ct, per, q["group"])
        out -= origin.permute(0, 2, 1, 3)[..., None]
        out *= scale.permute(0, 2, 1, 3)[..., None]
        return out.view(rt * 16, ct * 128)[:q["rows"], :q["cols"]]

    def act(g):
        if case["act"] == "silu":
            return g * torch.sigmoid(g)
        return 0.5 * g * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (g + 0.044715 * g ** 3)))

    if op in ("norm", "ffn"):
        h = s["x"].double() + s["residual"].double()
        rstd = (h.square().sum(1, True) / case["cols"] + s["eps"]).rsqrt()
        if op == "norm" and not case["eight"]:
            return h, h * s["weight"].double() * rstd
        # the definition quantises the binary32 product of the binary32 sum and the weight
        p = (h.float() * s["weight"].float()).double()
        most = p.abs().amax(1, True)
        x = torch.round(p * 127.0 / most) * (most * rstd / 127.0)
        if op == "norm":
            return h, x
        hidden = act(x @ matrix(s["gate"]).t()) * (x @ matrix(s["up"]).t())
        return h, hidden @ matrix(s["down"]).t()
    x = s["x"].double()
    if s["x_scale"] is not None:
        x = x * s["x_scale"].double()[:, None]
    if op == "matvec":
        return x @ matrix(s["q"]).t()
    return act(x @ matrix(s["gate"]).t()) * (x @ matrix(s["up"]).t())
