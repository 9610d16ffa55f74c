"""Cases for timing the dense-parameter operators: the AdamW step over many tensors with FP32 or 8-bit states, the global
gradient norm with its clipping factor, and the conversion of a state between the two forms.

`run` computes each operator either in elementary torch operations (`own` false) or through the library's DensePlan
(`own` true).  All tensors of a case live in a few flat buffers, as in programs that shard or checkpoint them flat; an
operator works on per-tensor views of them.  8-bit states are blocks of 256 elements: E4M3 values of m and of
r = sqrt(v), and one power-of-two scale for each of the two per block."""
import math
import random

import numpy as np
import torch

own = False

BLOCK = 256
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def f32(x):
    return float(np.float32(x))


# ---- the tensors of a case ------------------------------------------------------------------------------------------

def shapes_of(case):
    """(rows, columns) of every tensor of the case."""
    if case["set"] == "llama":       # a decoder's matrices, its normalisation weights and its embedding
        h, f = case["hidden"], case["ffn"]
        layer = [(h, h)] * 4 + [(f, h), (f, h), (h, f)] + [(1, h)] * 2
        return layer * case["layers"] + [(1, h)] + ([(case["vocab"], h)] if case["vocab"] else [])
    if case["set"] == "vectors":     # normalisation weights alone
        return [(1, case["width"])] * case["tensors"]
    rng = random.Random(case["shape_seed"])   # ragged: sizes over three orders of magnitude that add up to `elements`
    part = [math.exp(rng.uniform(0.0, math.log(1000.0))) for _ in range(case["tensors"])]
    sizes = [max(1, int(case["elements"] * p / sum(part))) for p in part]
    return [(1, n) if n < 64 or rng.random() < 0.3 else (lambda r: (r, max(1, n // r)))(rng.randint(2, max(2, int(math.sqrt(n))))) for n in sizes]


def layout_of(case):
    """Per tensor (rows, columns, pitch, offset) in the flat parameter and gradient buffers, and their length.
    aligned: every tensor starts at a multiple of 256 elements; packed: directly behind the one before; pitched: rows
    padded to a multiple of 8 elements, as the library's own matrices are."""
    at, out = 0, []
    for r, c in shapes_of(case):
        ld = (c + 7) // 8 * 8 if case["layout"] == "pitched" and r > 1 else c
        out.append((r, c, ld, at))
        at += r * ld
        if case["layout"] != "packed":
            at = (at + BLOCK - 1) // BLOCK * BLOCK
    return out, at


def blocks_of(shapes):
    return [(r * c + BLOCK - 1) // BLOCK for r, c in shapes]


# ---- 8-bit blocks in elementary operations ----------------------------------------------------------------------------

def scales_of(x):
    """x: blocks x 256, non-negative.  The smallest power of two s with max x <= 448 s, and 1 / s."""
    bits = x.amax(dim=1, keepdim=True).view(torch.int32)
    e = (((bits + 0x1FFFFF) >> 23) - 135).clamp(min=-126)
    return ((e + 127) << 23).view(torch.float32), ((127 - e) << 23).view(torch.float32)


def random_words(counter, key1, key2):
    """32 random bits for each counter: a multiply-xorshift mix of 32-bit words in 64-bit integers."""
    m = 0xFFFFFFFF
    x = (counter + key1) & m
    x = x ^ (x >> 16)
    x = (x * 0x85EBCA6B) & m
    x = x ^ (x >> 13) ^ key2
    x = (x * 0xC2B2AE35) & m
    return x ^ (x >> 16)


def mix32(x):
    m = 0xFFFFFFFF
    x &= m
    x ^= x >> 16
    x = (x * 0x85EBCA6B) & m
    x ^= x >> 13
    x = (x * 0xC2B2AE35) & m
    return x ^ (x >> 16)


def keys_of(seed, step, tensor):
    """The two 32-bit keys of one tensor's random words in one step."""
    k1 = mix32(mix32((seed & 0xFFFFFFFF) ^ mix32((seed >> 32) + 0x9E3779B9)) ^ mix32((step & 0xFFFFFFFF) + 0x7F4A7C15 * (tensor + 1)))
    return k1, mix32(k1 ^ 0xA511E9B3)


def to_e4m3(y, bits16=None):
    """|y| <= 448 to E4M3, to nearest even, or up with the probability of the remainder (16 random bits)."""
    if bits16 is None:
        return y.to(torch.float8_e4m3fn)
    a = y.abs()
    c = torch.where(a < 2.0 ** -6, 2.0 ** -6, 0.0)
    z = (a + c).view(torch.int32) + (bits16.to(torch.int32) << 4)
    a = (z & -0x100000).view(torch.float32) - c
    return torch.where(y < 0, -a, a).to(torch.float8_e4m3fn)


def encode(m, r, bits=None):
    """Blocks of m and r as codes and scales; a root above zero is not stored as zero.  bits: 32 random bits per element."""
    sm, im = scales_of(m.abs())
    sr, ir = scales_of(r)
    lo, hi = (None, None) if bits is None else (bits & 0xFFFF, bits >> 16)
    cm, cr = to_e4m3(m * im, lo), to_e4m3(r * ir, hi).float()
    cr = torch.where(r > 0, cr.clamp(min=2.0 ** -9), cr).to(torch.float8_e4m3fn)
    return cm, cr, torch.cat([sm, sr], dim=1)


# ---- cases --------------------------------------------------------------------------------------------------------------

LLAMA_60M = dict(set="llama", layers=8, hidden=512, ffn=1376, vocab=32000)
LLAMA_130M = dict(set="llama", layers=12, hidden=768, ffn=2048, vocab=32000)
LLAMA_350M = dict(set="llama", layers=24, hidden=1024, ffn=2736, vocab=32000)
LLAMA_1B = dict(set="llama", layers=24, hidden=2048, ffn=5461, vocab=32000)


def listed():
    step32 = dict(op="step", state="f32", stochastic=False, steps=100)
    step8 = dict(op="step", state="q8", steps=100)
    return [
        # the normalisation weights of the 60M model next to TSR blocks: the smallest call, all latency
        dict(step32, name="f32_norm_weights_60m", set="vectors", tensors=17, width=512, layout="aligned", p="f32", g="f32", image=False, clip=False),
        # AdamW baseline of the 60M model: FP32 masters, BF16 gradients, clipping, and the BF16 weights the model runs on
        dict(**step32, **LLAMA_60M, name="f32_60m_image", layout="aligned", p="f32", g="bf16", image=True, clip=True),
        # parameters packed one behind the other in a flat buffer, odd sizes: hardly a tensor starts on 16 bytes
        dict(step32, name="f32_packed_ragged", set="ragged", tensors=61, elements=24_000_000, shape_seed=5, layout="packed", p="bf16", g="bf16", image=False, clip=True),
        # AdamW baseline of the 1B model, the largest call: FP32 masters and BF16 gradients
        dict(**step32, **LLAMA_1B, name="f32_1b", layout="aligned", p="f32", g="bf16", image=False, clip=True),
        # one layer's vectors with 8-bit states: the smallest call
        dict(step8, name="q8_vectors", set="vectors", tensors=9, width=2048, layout="aligned", p="bf16", g="bf16", image=False, clip=False, stochastic=False),
        # the 130M model in BF16 with 8-bit states, rounded to nearest
        dict(**step8, **LLAMA_130M, name="q8_130m", layout="aligned", p="bf16", g="bf16", image=False, clip=True, stochastic=False),
        # two layers of the 1B model as the library holds its matrices: rows of 5461 at a pitch of 5464
        dict(**step8, **dict(LLAMA_1B, layers=2, vocab=0), name="q8_1b_layers_pitched", layout="pitched", p="f32", g="bf16", image=False, clip=True, stochastic=True),
        # the 1B model in BF16 with 8-bit states and stochastic rounding, as a memory-bound user runs it
        dict(**step8, **LLAMA_1B, name="q8_1b_stochastic", layout="aligned", p="bf16", g="bf16", image=False, clip=True, stochastic=True),
        # clipping factor of a few vectors: latency
        dict(op="norm", name="norm_vectors", set="vectors", tensors=17, width=512, layout="aligned", g="f32"),
        # clipping factor of the whole 1B gradient
        dict(LLAMA_1B, op="norm", name="norm_1b", layout="aligned", g="bf16"),
        # a checkpoint with FP32 moments loaded into a run with 8-bit states
        dict(LLAMA_350M, op="encode", name="encode_350m", layout="aligned"),
        # 8-bit states written out as FP32 moments, odd sizes
        dict(op="decode", name="decode_ragged", set="ragged", tensors=37, elements=30_000_000, shape_seed=9, layout="aligned"),
    ]


def draw(rng):
    op = rng.choice(["step", "step", "step", "step", "step", "norm", "encode", "decode"])
    layout = rng.choice(["aligned", "aligned", "packed", "pitched"]) if op in ("step", "norm") else "aligned"
    top = 1.1e9 if layout == "aligned" else 6e7
    elements = int(math.exp(rng.uniform(math.log(300.0), math.log(top))))
    case = dict(op=op, set="ragged", tensors=rng.randint(1, max(1, min(200, elements // 50))), elements=elements,
                shape_seed=rng.randint(1, 10 ** 6), layout=layout)
    if op in ("step", "norm"):
        case["g"] = rng.choice(["bf16", "bf16", "f32"])
    if op == "step":
        case["state"] = rng.choice(["f32", "q8", "q8"])
        case["p"] = rng.choice(["bf16", "f32"])
        case["image"] = case["p"] == "f32" and rng.random() < 0.4
        case["clip"] = rng.random() < 0.7
        case["stochastic"] = rng.random() < 0.5
        case["steps"] = int(math.exp(rng.uniform(0.0, math.log(1e5))))
        # the listed 1B call with FP32 masters stays the largest
        each = work(case)["bytes"] / sum(r * c for r, c in shapes_of(case))
        case["elements"] = min(elements, int(33e9 / each))
    return case


def work(case):
    shapes = shapes_of(case)
    n, nb = sum(r * c for r, c in shapes), sum(blocks_of(shapes))
    if case["op"] == "norm":
        return {"bytes": n * SIZE[case["g"]] + 8, "flops": 2 * n}
    if case["op"] in ("encode", "decode"):
        return {"bytes": n * 10 + nb * 8, "flops": 6 * n}
    state = 16 * n if case["state"] == "f32" else 4 * n + 16 * nb
    image = 2 * n if case["image"] else 0
    return {"bytes": state + n * (2 * SIZE[case["p"]] + SIZE[case["g"]]) + image, "flops": (16 if case["state"] == "f32" else 24) * n}


# ---- inputs ---------------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    tensors, total = layout_of(case)
    shapes = [(r, c) for r, c, _, _ in tensors]
    per = blocks_of(shapes)
    nb = sum(per)
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    rng = random.Random(seed)
    step = case.get("steps", 1)
    s = dict(case=case, seed=seed, tensors=tensors, nb=nb, step=step,
             lr=f32(10.0 ** rng.uniform(-4, -2.5)), wd=f32(0.1), b1=f32(0.9), b2=f32(rng.choice([0.95, 0.999])), eps=f32(1e-8),
             rseed=rng.getrandbits(64) >> 1)
    starts = np.concatenate([[0], np.cumsum(per)])
    s["first"] = [int(x) for x in starts[:-1]]        # first block of every tensor in the state buffers

    # where element i of the state (tensors padded to whole blocks) lies in the flat buffers; the place behind the last
    # element stands for padding.  Not needed where the flat buffers have the state's own layout.
    s["pos"] = None
    if case["op"] in ("step", "norm") and case["layout"] != "aligned":
        pos = torch.full((nb * BLOCK,), total, dtype=torch.int64, device=dev)
        for (r, c, ld, at), b in zip(tensors, s["first"]):
            i = torch.arange(r * c, device=dev)
            pos[b * BLOCK: b * BLOCK + r * c] = i // c * ld + i % c + at
        s["pos"] = pos.view(nb, BLOCK)
        s["src"] = (pos < total).nonzero().view(-1)
        s["dst"] = pos[s["src"]]
    elif case["op"] in ("step", "norm"):
        total = nb * BLOCK
    s["total"] = total

    counts = torch.tensor(per, device=dev)
    tail = torch.tensor([r * c - (b - 1) * BLOCK for (r, c), b in zip(shapes, per)], device=dev)
    valid = torch.full((nb,), BLOCK, device=dev)
    valid[torch.cumsum(counts, 0) - 1] = tail
    tail_blocks = (valid < BLOCK).nonzero().view(-1)
    off = torch.arange(BLOCK, device=dev)[None, :] >= valid[tail_blocks, None]

    def clear(x):     # zero in the places that pad a tensor's last block
        x[tail_blocks] = torch.where(off, torch.zeros((), dtype=x.dtype, device=dev), x[tail_blocks])
        return x

    # gradients of one run: each block of 256 has a size of its own, and some (rows of tokens that did not occur) are zero
    sigma = torch.exp(torch.randn(nb, 1, generator=gen, device=dev) * 1.5 - 7.0)
    sigma *= torch.rand(nb, 1, generator=gen, device=dev) > 0.05

    def flat(x, dtype):   # blocks -> a flat buffer in the case's layout
        if s["pos"] is None:
            return x.to(dtype)
        y = torch.zeros(total + 1, dtype=dtype, device=dev)
        y[s["dst"]] = x.view(-1)[s["src"]].to(dtype)
        return y

    if case["op"] in ("step", "norm"):
        s["grad"] = flat(clear(torch.randn(nb, BLOCK, generator=gen, device=dev) * sigma), DT[case["g"]])
    if case["op"] == "step":
        s["param"] = flat(clear(torch.randn(nb, BLOCK, generator=gen, device=dev) * 0.02), DT[case["p"]])
        if case["image"]:
            s["image"] = torch.zeros_like(s["param"], dtype=torch.bfloat16)
        # vectors are not decayed; matrices with few rows learn at half the rate
        wdm = [0.0 if r == 1 else 1.0 for r, c in shapes]
        lrm = [0.5 if 1 < r < 16 else 1.0 for r, c in shapes]
        s["wd_mult"], s["lr_mult"] = wdm, lrm
        rep = lambda v: torch.tensor(v, dtype=torch.float32, device=dev).repeat_interleave(counts)[:, None]  # noqa: E731
        lr = s["lr"] * rep(lrm)
        s["lr_block"], s["decay_block"] = lr, 1.0 - lr * (s["wd"] * rep(wdm))
        s["clip"] = torch.tensor([rng.uniform(0.2, 1.0)], device=dev) if case["clip"] else None
        if case["stochastic"]:
            keys = np.array([keys_of(s["rseed"], step, t) for t in range(len(shapes))], dtype=np.int64)
            s["key1"], s["key2"] = (torch.from_numpy(np.ascontiguousarray(keys[:, k])).to(dev).repeat_interleave(counts)[:, None] for k in (0, 1))
            s["within"] = (torch.arange(nb, device=dev) - torch.tensor(s["first"], device=dev).repeat_interleave(counts))[:, None] * BLOCK
    if case["op"] != "norm":
        m = clear(torch.randn(nb, BLOCK, generator=gen, device=dev) * (0.3 * sigma))
        v = clear((torch.rand(nb, BLOCK, generator=gen, device=dev) + 0.5) * sigma).square_()
        if case["op"] == "decode" or case.get("state") == "q8":
            s["m8"], s["r8"], s["scale"] = encode(m, v.sqrt())
        if case["op"] in ("encode", "decode") or case.get("state") == "f32":
            s["m"], s["v"] = m, v
        if case["op"] == "decode":
            s["m"], s["v"] = torch.zeros_like(m), torch.zeros_like(v)
        if case["op"] == "encode":
            s["m8"], s["r8"] = (torch.zeros(nb, BLOCK, dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn) for _ in range(2))
            s["scale"] = torch.zeros(nb, 2, device=dev)
    if own:
        make_plans(s)
    return s


def make_plans(s):
    import paper_2602_08007_b200 as tsr
    case = s["case"]

    def matrices(flat):   # per-tensor views of a flat buffer
        x = flat.view(-1)
        return [torch.as_strided(x, (r, c), (ld, 1), at) for r, c, ld, at in s["tensors"]]

    def state(*names):    # per-tensor views of state buffers
        rows = [(r * c, b) for (r, c, _, _), b in zip(s["tensors"], s["first"])]
        return [[s[k].view(-1)[b * BLOCK: b * BLOCK + n] for n, b in rows] if k != "scale" else
                [s[k][b: b + (n + BLOCK - 1) // BLOCK] for n, b in rows] for k in names]

    if case["op"] == "norm":
        s["plan"] = tsr.DensePlan(None, matrices(s["grad"]))
    elif case["op"] == "step":
        st = state("m", "v") if case["state"] == "f32" else state("m8", "r8", "scale")
        s["plan"] = tsr.DensePlan(matrices(s["param"]), matrices(s["grad"]), states=list(zip(*st)), images=matrices(s["image"]) if case["image"] else None,
                                  lr_mult=s["lr_mult"], wd_mult=s["wd_mult"])
    else:
        s["plan32"] = tsr.DensePlan(None, None, states=list(zip(*state("m", "v"))))
        s["plan8"] = tsr.DensePlan(None, None, states=list(zip(*state("m8", "r8", "scale"))))
    s["tsr"] = tsr


# ---- one pass ---------------------------------------------------------------------------------------------------------------

MAX_NORM = 1.0


def run(s):
    return (own_pass if own else plain_pass)(s)


def own_pass(s):
    case, tsr = s["case"], s["tsr"]
    if case["op"] == "norm":
        return s["plan"].grad_norm(MAX_NORM)
    if case["op"] == "encode":
        s["plan8"].copy_state(s["plan32"])
        return s["m8"], s["r8"], s["scale"]
    if case["op"] == "decode":
        s["plan32"].copy_state(s["plan8"])
        return s["m"], s["v"]
    hyper = tsr.make_hyper(s["step"], lr=s["lr"], beta1=s["b1"], beta2=s["b2"], eps=s["eps"], weight_decay=s["wd"])
    s["plan"].step(hyper, grad_scale=s["clip"], rounding=tsr.TSR_ROUND_STOCHASTIC if case["stochastic"] else tsr.TSR_ROUND_NEAREST, seed=s["rseed"])
    return outputs(s)


def outputs(s):
    out = {"param": s["param"]}
    if s["case"]["image"]:
        out["image"] = s["image"]
    for k in ("m", "v") if s["case"]["state"] == "f32" else ("m8", "r8", "scale"):
        out[k] = s[k]
    return out


def blocks(s, flat):
    """A flat buffer as blocks of 256 in 32 bits."""
    return (flat if s["pos"] is None else flat[s["pos"]]).float()


def store(s, flat, x):
    if s["pos"] is None:
        flat.copy_(x)
    else:
        flat[s["dst"]] = x.view(-1)[s["src"]].to(flat.dtype)


def plain_pass(s):
    case = s["case"]
    if case["op"] == "norm":
        g = s["grad"].float()
        n = (g * g).sum().sqrt()
        return torch.stack([n, (MAX_NORM / (n + 1e-6)).clamp(max=1.0)])
    if case["op"] == "encode":
        m8, r8, scale = encode(s["m"], s["v"].sqrt())
        s["m8"].copy_(m8), s["r8"].copy_(r8), s["scale"].copy_(scale)
        return s["m8"], s["r8"], s["scale"]
    if case["op"] == "decode":
        s["m"].copy_(s["m8"].float() * s["scale"][:, :1])
        r = s["r8"].float() * s["scale"][:, 1:]
        s["v"].copy_(r * r)
        return s["m"], s["v"]
    b1, b2, t = s["b1"], s["b2"], s["step"]
    g = blocks(s, s["grad"])
    if s["clip"] is not None:
        g = g * s["clip"]
    bits = None
    if case["stochastic"]:
        e = s["within"] + torch.arange(BLOCK, device=g.device)
        bits = random_words(e, s["key1"], s["key2"]) if case["state"] == "q8" else None
        if case["p"] == "bf16":
            w = random_words(e >> 1, s["key1"] ^ 0x5BD1E995, s["key2"])
            p_bits = torch.where((e & 1) == 1, w >> 16, w & 0xFFFF).to(torch.int32)
            del w
        del e
    if case["state"] == "f32":
        m, v = s["m"], s["v"]
    else:
        m, r = s["m8"].float() * s["scale"][:, :1], s["r8"].float() * s["scale"][:, 1:]
        v = r * r
        del r
    m = m * b1 + g * f32(1.0 - b1)
    v = v * b2 + (g * g) * f32(1.0 - b2)
    del g
    if case["state"] == "f32":
        s["m"].copy_(m), s["v"].copy_(v)
        d = (m * f32(1.0 / (1.0 - b1 ** t))) / ((v * f32(1.0 / (1.0 - b2 ** t))).sqrt() + s["eps"])
    else:
        r = v.sqrt()
        m8, r8, scale = encode(m, r, bits)
        del bits
        s["m8"].copy_(m8), s["r8"].copy_(r8), s["scale"].copy_(scale)
        d = (m * f32(1.0 / (1.0 - b1 ** t))) / (r * f32(math.sqrt(1.0 / (1.0 - b2 ** t))) + s["eps"])
        del r, m8, r8
    del m, v
    p = blocks(s, s["param"]) * s["decay_block"] - s["lr_block"] * d
    if case["stochastic"] and case["p"] == "bf16":
        p = ((p.view(torch.int32) + p_bits) & -0x10000).view(torch.float32)
    store(s, s["param"], p)
    if case["image"]:
        store(s, s["image"], p)
    return outputs(s)


# ---- the definition in 64 bits ------------------------------------------------------------------------------------------------

def exact(case, seed):
    global own
    held, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = held
    if case["op"] == "norm":
        parts = [x.double().square().sum() for x in s["grad"].view(-1).split(1 << 26)]
        n = torch.stack(parts).sum().sqrt()
        return torch.stack([n, torch.minimum(torch.ones_like(n), MAX_NORM / (n + 1e-6))])
    slab = 1 << 18   # blocks at a time

    def in_slabs(fn):   # fn(a, b): outputs of blocks a to b, joined
        parts = [fn(a, min(a + slab, s["nb"])) for a in range(0, s["nb"], slab)]
        return [torch.cat([p[k] for p in parts]) for k in range(len(parts[0]))]

    def values(x, a, b):
        return x[a:b].double()

    def scale64(x):      # smallest power of two s with max x <= 448 s
        e = torch.ceil(torch.log2(x.amax(dim=1, keepdim=True).clamp(min=1e-300) / 448.0)).clamp(min=-126)
        return torch.pow(torch.full_like(e, 2.0), e)

    if case["op"] == "encode":
        def enc(a, b):
            m, r = values(s["m"], a, b), values(s["v"], a, b).sqrt()
            sm, sr = scale64(m.abs()), scale64(r)
            return m / sm, r / sr, torch.cat([sm, sr], dim=1)
        return tuple(in_slabs(enc))
    if case["op"] == "decode":
        return tuple(in_slabs(lambda a, b: (values(s["m8"], a, b) * s["scale"][a:b, :1].double(),
                                            (values(s["r8"], a, b) * s["scale"][a:b, 1:].double()) ** 2)))
    b1, b2, t = s["b1"], s["b2"], s["step"]
    lr_mult = torch.tensor(s["lr_mult"], dtype=torch.float64, device="cuda")
    wd_mult = torch.tensor(s["wd_mult"], dtype=torch.float64, device="cuda")
    which = torch.repeat_interleave(torch.arange(len(s["tensors"]), device="cuda"),
                                    torch.tensor(blocks_of([(r, c) for r, c, _, _ in s["tensors"]]), device="cuda"))
    clip = 1.0 if s["clip"] is None else float(s["clip"].double())

    def flat64(x, a, b):
        return values(x, a, b) if s["pos"] is None else x[s["pos"][a:b]].double()

    def one(a, b):
        g = flat64(s["grad"], a, b) * clip
        if case["state"] == "f32":
            m, v = values(s["m"], a, b), values(s["v"], a, b)
        else:
            m = values(s["m8"], a, b) * s["scale"][a:b, :1].double()
            v = (values(s["r8"], a, b) * s["scale"][a:b, 1:].double()) ** 2
        m = b1 * m + (1.0 - b1) * g
        v = b2 * v + (1.0 - b2) * g * g
        d = m / (1.0 - b1 ** t) / ((v / (1.0 - b2 ** t)).sqrt() + s["eps"])
        lr = s["lr"] * lr_mult[which[a:b], None]
        p = flat64(s["param"], a, b) * (1.0 - lr * s["wd"] * wd_mult[which[a:b], None]) - lr * d
        if case["state"] == "f32":
            return p, m, v
        r = v.sqrt()
        sm, sr = scale64(m.abs()), scale64(r)
        return p, m / sm, r / sr, torch.cat([sm, sr], dim=1)

    p, *state = in_slabs(one)
    if s["pos"] is not None:
        q = torch.zeros(s["total"] + 1, dtype=torch.float64, device="cuda")
        q[s["dst"]] = p.view(-1)[s["src"]]
        p = q
    out = {"param": p}
    if case["image"]:
        out["image"] = p
    out.update(zip(("m", "v") if case["state"] == "f32" else ("m8", "r8", "scale"), state))
    return out
