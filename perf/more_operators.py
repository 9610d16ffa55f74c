"""Cases for timing the layer operators: the norm over rows (with or without the mean) forward and backward, the linear layer
with bias, activation, dropout and residual in its epilogue forward and backward, and dropout on its own.

`run` computes each operator either in elementary torch operations (`own` false) or through the library's calls (`own` true).
Token matrices have one row per token.  Widths are those of the decoders whose gradients the library steps; rows of 5461 BF16
entries are no multiple of 16 bytes, and the library's own gradient matrices then have a pitch of 5464."""
import math
import random

import numpy as np
import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
EPS = 1e-5


def listed():
    norm = dict(op="norm", center=True, bias=True)
    lin = dict(op="linear", act="none", bias=True, residual=False, p=0.0, pitched=False)
    return [
        # the tokens of one short sequence in the 60M decoder: the smallest call, all latency
        dict(norm, name="norm_fwd_short", dir="forward", rows=64, cols=512, dtype="bf16"),
        # a training batch of the 1B decoder
        dict(norm, name="norm_fwd_1b", dir="forward", rows=16384, cols=2048, dtype="bf16"),
        # a batch of the 350M decoder in 32 bits, with the gradients of weight and bias
        dict(norm, name="norm_bwd_350m_f32", dir="backward", rows=8192, cols=1024, dtype="f32"),
        # a norm without mean over the feed-forward width of the 1B decoder, odd rows, odd number of them
        dict(norm, name="norm_bwd_1b_odd", dir="backward", rows=6007, cols=5461, dtype="bf16", center=False, bias=False),
        # one token through an output projection of the 1B decoder: the weight is read once
        dict(lin, name="linear_fwd_one_token", dir="forward", rows=1, ins=2048, outs=2048, dtype="bf16", residual=True),
        # up projection of the 130M decoder, a ragged batch, the pre-activations kept for the backward pass
        dict(lin, name="linear_fwd_130m_gelu", dir="forward", rows=5003, ins=768, outs=2048, dtype="bf16", act="gelu"),
        # down projection of the 1B decoder with dropout and residual; rows of 5461 entries, back to back
        dict(lin, name="linear_fwd_1b_down", dir="forward", rows=8192, ins=5461, outs=2048, dtype="bf16", p=0.1, residual=True),
        # gate projection of the 1B decoder, backward, into a gradient matrix of the library: the largest call
        dict(lin, name="linear_bwd_1b_gate", dir="backward", rows=8192, ins=2048, outs=5461, dtype="bf16", act="silu", bias=False, pitched=True),
        # attention output of the 60M decoder over many tokens, with dropout: small matrices, a long sum for the weight's gradient
        dict(lin, name="linear_bwd_60m_long", dir="backward", rows=32768, ins=512, outs=512, dtype="bf16", p=0.1),
        # gate projection of the 60M decoder in 32 bits
        dict(lin, name="linear_bwd_60m_f32", dir="backward", rows=4096, ins=512, outs=1376, dtype="f32"),
        # dropout on the embeddings of a short sequence
        dict(op="dropout", name="dropout_short", rows=64, cols=512, dtype="bf16", p=0.1, residual=False),
        # dropout and residual of a training batch of the 1B decoder
        dict(op="dropout", name="dropout_1b", rows=32768, cols=2048, dtype="bf16", p=0.1, residual=True),
    ]


def spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "linear", "linear", "linear", "dropout"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    case = dict(op=op, rows=spread(rng, 1, 32768), dtype=dtype)
    if op == "linear":
        even = rng.choice([1, 8, 64])         # any width, whole vectors, whole blocks of a tile
        for k in ("ins", "outs"):
            case[k] = max(1, spread(rng, 24, 8192) // even) * even
        case.update(dir=rng.choice(["forward", "backward"]), act=rng.choice(["none", "none", "relu", "gelu", "gelu_tanh", "silu"]),
                    bias=rng.random() < 0.6, residual=rng.random() < 0.5, p=rng.choice([0.0, 0.0, 0.1, 0.5]), pitched=rng.random() < 0.5)
        top = (350e9 if case["dir"] == "backward" else 175e9) * (0.1 if dtype == "f32" else 1.0)
        case["rows"] = max(1, min(case["rows"], int(top / (2 * case["ins"] * case["outs"]))))
        return case
    case["cols"] = spread(rng, 16, 12000)
    case["rows"] = max(1, min(case["rows"], int(1.2e8 / case["cols"])))
    if op == "norm":
        case.update(dir=rng.choice(["forward", "backward"]), center=rng.random() < 0.5, bias=rng.random() < 0.5)
    else:
        case.update(p=rng.choice([0.05, 0.1, 0.5]), residual=rng.random() < 0.5)
    return case


def work(case):
    e, r = SIZE[case["dtype"]], case["rows"]
    if case["op"] == "norm":
        n = r * case["cols"]
        vec = 4 * case["cols"] * (2 if case["bias"] else 1)
        if case["dir"] == "forward":
            return {"bytes": 2 * n * e + vec + 8 * r, "flops": 8 * n}
        return {"bytes": 3 * n * e + vec + 4 * case["cols"] + 8 * r, "flops": 14 * n}
    if case["op"] == "dropout":
        n = r * case["cols"]
        return {"bytes": n * e * (3 if case["residual"] else 2), "flops": 3 * n}
    i, o = case["ins"], case["outs"]
    kept = r * o if case["act"] != "none" else 0                     # pre-activations: written forward, read backward
    if case["dir"] == "forward":
        return {"bytes": e * (r * i + i * o + r * o * (2 if case["residual"] else 1) + kept), "flops": 2 * r * i * o}
    return {"bytes": e * (r * o + kept + 2 * r * i + 2 * i * o), "flops": 4 * r * i * o}


# ---- inputs -------------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    rng = random.Random(seed)
    dt, r = DT[case["dtype"]], case["rows"]
    s = dict(case=case)

    def normal(*shape, sigma=1.0, dtype=dt):
        return (torch.randn(*shape, generator=gen, device=dev) * sigma).to(dtype)

    def activations(n):       # channels of different size, a few of them large, and an offset
        size = torch.exp(0.5 * torch.randn(n, generator=gen, device=dev))
        size[torch.rand(n, generator=gen, device=dev) < 0.01] *= 8.0
        return ((torch.randn(r, n, generator=gen, device=dev) + 0.2) * size).to(dt)

    if case.get("p"):
        s["seed"], s["offset"] = rng.getrandbits(63), rng.getrandbits(40)
    if case["op"] == "norm":
        n = case["cols"]
        s["x"] = activations(n)
        s["w"] = 1.0 + normal(n, sigma=0.1, dtype=torch.float32)
        s["b"] = normal(n, sigma=0.1, dtype=torch.float32) if case["bias"] else None
        if case["dir"] == "backward":
            s["dy"] = normal(r, n, sigma=1e-2)
            x = s["x"].double()
            mean = x.mean(1) if case["center"] else torch.zeros(r, device=dev, dtype=torch.float64)
            var = (x - mean[:, None]).square_().mean(1)
            s["stats"] = torch.stack([mean, (var + EPS).rsqrt()], dim=1).float()
    elif case["op"] == "dropout":
        s["x"] = normal(r, case["cols"])
        s["res"] = normal(r, case["cols"]) if case["residual"] else None
    else:
        i, o = case["ins"], case["outs"]
        s["x"] = normal(r, i)
        s["w"] = normal(o, i, sigma=0.02)
        s["b"] = normal(o, sigma=0.1, dtype=torch.float32) if case["bias"] else None
        s["res"] = normal(r, o) if case["residual"] and case["dir"] == "forward" else None
        if case["dir"] == "backward":
            s["dy"] = normal(r, o, sigma=1e-2)
            s["pre"] = normal(r, o) if case["act"] != "none" else None
            ld = (i + 7) // 8 * 8 if case["pitched"] else i
            s["G"] = torch.zeros(o, ld, dtype=dt, device=dev)[:, :i]    # the bound gradient matrix of the optimizer's plan
            s["gb"] = torch.zeros(o, dtype=torch.float32, device=dev) if case["bias"] else None
    if own:
        import paper_2602_08007_b200 as tsr
        s["tsr"] = tsr
        s["drop"] = tsr.Dropout(case["p"], s["seed"], s["offset"]) if case.get("p") else None
    return s


# ---- the random words of dropout, and the activations ---------------------------------------------------------------------

M32 = 0xFFFFFFFF


def mix32(x):
    """Multiply-xorshift mixing of 32-bit words, held in 64-bit integers (or Python's own)."""
    x = x & M32
    x = x ^ (x >> 16)
    x = (x * 0x85EBCA6B) & M32
    x = x ^ (x >> 13)
    x = (x * 0xC2B2AE35) & M32
    return x ^ (x >> 16)


def call_key(seed, offset):
    k = mix32(mix32((seed & M32) ^ mix32((seed >> 32) + 0x9E3779B9)) ^ mix32((offset & M32) + 0x7F4A7C15))
    return mix32(k ^ (((offset >> 32) * 0x85EBCA77) & M32))


def kept(s, cols):
    """Which entries dropout keeps: 16 random bits of each against the threshold."""
    dev, rows = s["case_device"], s["case"]["rows"]
    row = torch.arange(rows, device=dev)[:, None]
    r1 = mix32(call_key(s["seed"], s["offset"]) ^ mix32((row & M32) + 0x9E3779B9 * ((row >> 32) + 1)))
    r2 = mix32(r1 ^ 0xA511E9B3)
    x = (torch.arange((cols + 1) // 2, device=dev)[None, :] + r1) & M32
    x ^= x >> 16
    x = x.mul_(0x85EBCA6B).bitwise_and_(M32)
    x ^= (x >> 13) ^ r2
    x = x.mul_(0xC2B2AE35).bitwise_and_(M32)
    x ^= x >> 16
    bits = torch.stack([x & 0xFFFF, x >> 16], dim=2).view(rows, -1)[:, :cols]
    return bits >= threshold(s["case"]["p"])


def threshold(p):
    return int(math.floor(p * 65536.0 + 0.5))


def factor(p):
    return 65536.0 / (65536 - threshold(p))


def dropped(s, x):
    if not s["case"].get("p"):
        return x
    s["case_device"] = x.device
    return torch.where(kept(s, x.shape[1]), x * factor(s["case"]["p"]), torch.zeros((), dtype=x.dtype, device=x.device))


def activation(kind, z):
    if kind == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if kind == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if kind == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if kind == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def slope(kind, z):
    """Derivative of the activation."""
    if kind == "relu":
        return (z > 0).to(z.dtype)
    if kind == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if kind == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
    t = 1.0 / (1.0 + torch.exp(-z))
    return t * (1.0 + z * (1.0 - t))


# ---- one pass -----------------------------------------------------------------------------------------------------------

def run(s):
    return (own_pass if own else plain_pass)(s)


def own_pass(s):
    case, tsr = s["case"], s["tsr"]
    if case["op"] == "norm":
        if case["dir"] == "forward":
            y, stats = tsr.norm_forward(s["x"], s["w"], s["b"], eps=EPS, center=case["center"])
            return {"y": y, "mean": stats[:, 0], "rstd": stats[:, 1]}
        dx, dw, db = tsr.norm_backward(s["dy"], s["x"], s["w"], s["stats"], center=case["center"], bias=case["bias"])
        return {"dx": dx, "dw": dw, "db": db}
    if case["op"] == "dropout":
        return {"y": tsr.dropout_forward(s["x"], s["drop"], residual=s["res"])}
    if case["dir"] == "forward":
        y, pre = tsr.linear_forward(s["x"], s["w"], s["b"], activation=case["act"], dropout=s["drop"], residual=s["res"], keep_pre=case["act"] != "none")
        return {"y": y, "pre": pre}
    dx, dw, db = tsr.linear_backward(s["dy"], s["x"], s["w"], pre=s["pre"], activation=case["act"], dropout=s["drop"], dweight=s["G"], dbias=s["gb"])
    return {"dx": dx, "dw": dw, "db": db}


def plain_pass(s):
    case, dt = s["case"], DT[s["case"]["dtype"]]
    x = s["x"].float()
    if case["op"] == "norm":
        if case["dir"] == "forward":
            mean = x.mean(1, keepdim=True) if case["center"] else torch.zeros(x.shape[0], 1, device=x.device)
            x = x - mean
            rstd = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
            y = x * rstd * s["w"]
            y = (y if s["b"] is None else y + s["b"]).to(dt)
            return {"y": y, "mean": mean[:, 0], "rstd": rstd[:, 0]}
        rstd, dy = s["stats"][:, 1:], s["dy"].float()
        h = (x - s["stats"][:, :1]) * rstd
        g = dy * s["w"]
        dx = g - h * (g * h).mean(1, keepdim=True)
        if case["center"]:
            dx -= g.mean(1, keepdim=True)
        return {"dx": (dx * rstd).to(dt), "dw": (dy * h).sum(0), "db": dy.sum(0) if case["bias"] else None}
    if case["op"] == "dropout":
        y = dropped(s, x)
        return {"y": (y if s["res"] is None else y + s["res"].float()).to(dt)}
    w = s["w"].float()
    if case["dir"] == "forward":
        z = x @ w.t()
        if s["b"] is not None:
            z += s["b"]
        y = dropped(s, activation(case["act"], z))
        if s["res"] is not None:
            y = y + s["res"].float()
        return {"y": y.to(dt), "pre": z.to(dt) if case["act"] != "none" else None}
    dz = dropped(s, s["dy"].float())
    if s["pre"] is not None:
        dz = dz * slope(case["act"], s["pre"].float())
    s["G"].copy_(dz.t() @ x)
    if s["gb"] is not None:
        torch.sum(dz, 0, out=s["gb"])
    return {"dx": (dz @ w).to(dt), "dw": s["G"], "db": s["gb"]}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------------

def exact_mask(s, rows, cols):
    """The factor of every entry, from unsigned 32-bit words on the host."""
    p = s["case"]["p"]

    def mix(a):
        a = a.copy()
        for shift, mul in ((16, 0x85EBCA6B), (13, 0xC2B2AE35)):
            a ^= a >> np.uint32(shift)
            a *= np.uint32(mul)
        return a ^ (a >> np.uint32(16))

    def word(v):
        return np.array([v % (1 << 32)], dtype=np.uint32)

    key = mix(word(s["seed"]) ^ mix(word((s["seed"] >> 32) + 0x9E3779B9))) ^ mix(word(s["offset"] % (1 << 32) + 0x7F4A7C15))
    key = mix(mix(key) ^ word((s["offset"] >> 32) * 0x85EBCA77))
    r1 = mix(key ^ mix(np.arange(rows, dtype=np.uint32) + np.uint32(0x9E3779B9)))
    r2 = mix(r1 ^ np.uint32(0xA511E9B3))
    c = np.arange((cols + 1) // 2, dtype=np.uint32)
    thr = min(65536, int(p * 65536 + 0.5))
    out = torch.empty(rows, cols, dtype=torch.float64, device="cuda")
    for at in range(0, rows, 4096):
        x = c[None, :] + r1[at:at + 4096, None]
        x ^= x >> np.uint32(16)
        x *= np.uint32(0x85EBCA6B)
        x = x ^ (x >> np.uint32(13)) ^ r2[at:at + 4096, None]
        x *= np.uint32(0xC2B2AE35)
        x ^= x >> np.uint32(16)
        halves = np.ascontiguousarray(x).view("<u2").reshape(x.shape[0], -1)[:, :cols]
        out[at:at + 4096] = torch.from_numpy((halves >= thr).astype(np.float32)).cuda().double() * (65536.0 / (65536 - thr))
    return out


def exact(case, seed):
    global own
    held, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = held
    rows = case["rows"]
    x = s["x"].double()
    if case["op"] == "norm":
        n = case["cols"]
        w = s["w"].double()
        if case["dir"] == "forward":
            mu = x.sum(1) / n if case["center"] else torch.zeros(rows, dtype=torch.float64, device="cuda")
            sd = torch.sqrt(torch.linalg.vector_norm(x - mu[:, None], dim=1) ** 2 / n + EPS)
            y = (x - mu[:, None]) / sd[:, None] * w[None, :]
            return {"y": y if s["b"] is None else y + s["b"].double(), "mean": mu, "rstd": 1.0 / sd}
        dy, mu, rstd = s["dy"].double(), s["stats"][:, 0].double(), s["stats"][:, 1].double()
        h = (x - mu[:, None]) * rstd[:, None]
        g = dy * w[None, :]
        c2 = torch.einsum("ij,ij->i", g, h) / n
        c1 = g.sum(1) / n if case["center"] else torch.zeros_like(c2)
        dx = (g - c1[:, None] - h * c2[:, None]) * rstd[:, None]
        return {"dx": dx, "dw": torch.einsum("ij,ij->j", dy, h), "db": dy.sum(0) if case["bias"] else None}
    if case["op"] == "dropout":
        y = x * exact_mask(s, rows, case["cols"])
        return {"y": y if s["res"] is None else y + s["res"].double()}
    w, kind = s["w"].double(), case["act"]
    mask = exact_mask(s, rows, case["outs"]) if case["p"] else 1.0
    normal = torch.distributions.Normal(torch.zeros((), dtype=torch.float64, device="cuda"), torch.ones((), dtype=torch.float64, device="cuda"))
    if case["dir"] == "forward":
        z = torch.matmul(x, w.transpose(0, 1))
        if s["b"] is not None:
            z = z + s["b"].double()[None, :]
        a = {"none": lambda: z, "relu": lambda: z.clamp(min=0.0), "gelu": lambda: z * normal.cdf(z), "silu": lambda: z * torch.sigmoid(z),
             "gelu_tanh": lambda: z * torch.sigmoid(2.0 * (2.0 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3))}[kind]()
        y = a * mask
        return {"y": y if s["res"] is None else y + s["res"].double(), "pre": z if kind != "none" else None}
    dz = s["dy"].double() * mask
    if kind != "none":
        z = s["pre"].double()
        g = torch.sigmoid(z)
        if kind == "relu":
            d = torch.where(z > 0, torch.ones_like(z), torch.zeros_like(z))
        elif kind == "gelu":
            d = normal.cdf(z) + z * torch.exp(normal.log_prob(z))
        elif kind == "silu":
            d = g + z * g * (1.0 - g)
        else:
            k = 2.0 * (2.0 / math.pi) ** 0.5
            g = torch.sigmoid(k * (z + 0.044715 * z ** 3))
            d = g + z * g * (1.0 - g) * k * (1.0 + 3.0 * 0.044715 * z ** 2)
        dz = dz * d
    return {"dx": torch.matmul(dz, w), "dw": torch.matmul(dz.transpose(0, 1), x), "db": dz.sum(0) if s["gb"] is not None else None}
