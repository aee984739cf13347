"""The timed operators at the two ends of a language-model worker's training step.

A step starts with the lookup of its tokens in the embedding table, and the gradient that comes back to
the table is a sum over equal tokens.  Before the gradients are used they are clipped by their norm over
all tensors, and a replica that is trained without compression takes an AdamW step over the list of its
tensors, with moments in 32 or in 8 bits.  Every case is one call of one of the four:

  lookup   out[t] = scale * W[token[t]]
  grad     dW[v] = scale * sum of dY[t] over the tokens t equal to v (or that, added to what dW holds)
  norm     the 2-norm N of all gradients and the factor min(1, max_norm / N)
  adamw    one AdamW step of many tensors, the gradients times a factor that lies on the device

The tensors of a model are consecutive pieces of flat vectors, as the rest of this framework keeps them.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
BETA1, BETA2, EPS = 0.9, 0.999, 1e-8
BLOCK = 256  # coordinates that share a scale of the 8-bit states

# ---------------------------------------------------------------------------------------------- cases
# lookup, grad: a table of vocab x dim (wtype), seqs sequences of length tokens (itype), whose frequencies
#   fall as rank^-skew; otype: the type of the output (lookup) or of dY (grad); pad: the table has a padding
#   token that takes no gradient; tied: the gradient is added to what the output head left in dW; shifted:
#   the tokens are all but the last of each sequence's length + 1 (the usual inputs of next-token training).
# norm, adamw: tensors: "" for one of d coordinates, "resnet18", "LxW" for L layers of width W (four matrices
#   and four vectors each), "LxW+V" for the same after a table of V x W, "odd:K" for K tensors of uneven, mostly
#   odd sizes, d in all; ptype, gtype: parameters and gradients; bits: of the states; copy: a bf16 copy of the
#   parameters is written too.


def _tokens(name, op, **kw):
    c = dict(op=op, vocab=50257, dim=1600, seqs=1, length=1, wtype="f32", otype="bf16", itype="i64", skew=1.0,
             pad=False, tied=False, shifted=False)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def _tensors(name, op, **kw):
    c = dict(op=op, tensors="", d=0, gtype="f32", ptype="f32", bits=32, copy=False, t=100, lr=1e-3, decay=0.1)
    c.update(kw)
    if op == "norm":
        c = {k: c[k] for k in ("op", "tensors", "d", "gtype")}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one new token: the latency of a lookup
        _tokens("lookup_one_token", "lookup", wtype="bf16"),
        # a worker's batch of the GPT-2-XL-sized model, out of 32-bit weights into 16-bit activations
        _tokens("lookup_16k", "lookup", seqs=16, length=1024, shifted=True),
        # one short sequence whose gradient joins that of a tied output head
        _tokens("grad_tied_384", "grad", vocab=30522, dim=768, length=384, otype="f32", tied=True),
        # the gradient of that batch, the whole table's gradient written in 32 bits
        _tokens("grad_16k", "grad", seqs=16, length=1024),
        # many tokens of few kinds with padding (short texts in a BERT-sized vocabulary): long sums
        _tokens("grad_256k_skewed", "grad", vocab=30522, dim=768, seqs=2048, length=127, skew=1.3, pad=True),
        # ResNet-18's 62 gradients
        _tensors("norm_resnet18", "norm", tensors="resnet18"),
        # a BERT-base-sized language model's 16-bit gradients
        _tensors("norm_bert_bf16", "norm", tensors="12x768+30522", gtype="bf16"),
        # the 500-dimensional problem: the latency of a step
        _tensors("adamw_toy_500", "adamw", d=500),
        # ResNet-18 in 32 bits
        _tensors("adamw_resnet18", "adamw", tensors="resnet18"),
        # the largest: 32-bit weights and states, 16-bit gradients, and the 16-bit copy that the model reads
        _tensors("adamw_355m_mixed", "adamw", tensors="24x1024+50257", gtype="bf16", copy=True),
        # 8-bit states with tensors of odd sizes and 32-bit weights
        _tensors("adamw8_odd_9m", "adamw", tensors="odd:40", d=9_000_001, bits=8),
        # 8-bit states where every byte counts: 16-bit weights and gradients, BERT-base-sized
        _tensors("adamw8_bert_bf16", "adamw", tensors="12x768+30522", ptype="bf16", gtype="bf16", bits=8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["lookup", "grad", "grad", "norm", "adamw", "adamw"])
    if op in ("lookup", "grad"):
        dim = _log_int(rng, 64, 1700)
        dim = rng.choice([dim, dim, -(-dim // 8) * 8, -(-dim // 64) * 64])
        vocab = min(_log_int(rng, 500, 130_000), 100_000_000 // dim)
        length = _log_int(rng, 1, 1024)
        seqs = max(1, min(_log_int(rng, 1, 512), 150_000_000 // (dim * length)))
        wtype, otype = rng.choice(["f32", "f32", "bf16", "f16"]), rng.choice(["f32", "bf16", "bf16", "f16"])
        return _tokens("", op, vocab=vocab, dim=dim, seqs=seqs, length=length, wtype=wtype, otype=otype,
                       itype=rng.choice(["i64", "i32"]), skew=rng.choice([0.0, 0.8, 1.0, 1.3]), pad=rng.random() < 0.3,
                       tied=op == "grad" and rng.random() < 0.4, shifted=rng.random() < 0.4)
    kind = rng.choice(["one", "layers", "odd", "odd"])
    kw = {}
    if kind == "one":
        kw.update(d=_log_int(rng, 1, 150_000_000))
    elif kind == "layers":
        kw.update(tensors="%dx%d" % (rng.randint(1, 24), 8 * _log_int(rng, 5, 100)))
    else:
        k = _log_int(rng, 2, 400)
        kw.update(tensors="odd:%d" % k, d=max(100 * k, _log_int(rng, 10_000, 60_000_000)))
    gtype = rng.choice(["f32", "bf16", "f16"])
    if op == "norm":
        return _tensors("", op, gtype=gtype, **kw)
    ptype = rng.choice(["f32", "f32", "bf16"])
    copy = ptype == "f32" and rng.random() < 0.4
    return _tensors("", op, gtype=gtype, ptype=ptype, bits=rng.choice([8, 32]), copy=copy,
                    t=rng.choice([0, 1, 10, 1000, 100_000]), lr=10.0 ** rng.randint(-5, -2),
                    decay=rng.choice([0.0, 0.01, 0.1]), **kw)


# ---------------------------------------------------------------------------------- a case's parts

def _sizes(case):
    kind = case["tensors"]
    if not kind:
        return [case["d"]]
    if kind == "resnet18":
        sizes, width = [64 * 147, 64, 64], 64
        for ch in (64, 128, 256, 512):
            sizes += [ch * width * 9, ch, ch, ch * ch * 9, ch, ch]
            sizes += [ch * width, ch, ch] if ch > 64 else []
            sizes += [ch * ch * 9, ch, ch] * 2
            width = ch
        return sizes + [512 * 1000, 1000]
    if kind.startswith("odd:"):
        k, d = int(kind[4:]), case["d"]
        share = [(0.02 + ((i + 1) * 0.6180339887) % 1.0) ** 4 for i in range(k)]
        sizes = [max(1, int(s / sum(share) * (d - k)) | 1) for s in share[:-1]]
        return sizes + [max(1, d - sum(sizes))]
    layers, width = kind.split("+")[0].split("x")
    layers, w = int(layers), int(width)
    table = [int(kind.split("+")[1]) * w] if "+" in kind else []
    return table + [3 * w * w, w * w, 4 * w * w, 4 * w * w, w, w, w, w] * layers


def _gen(seed, what):
    return torch.Generator(device="cuda").manual_seed(1 + 64 * (int(seed) % (1 << 40)) + what)


def _randn(n, seed, what, std=1.0, dtype=torch.float32):
    return torch.randn(n, generator=_gen(seed, what), device="cuda", dtype=dtype).mul_(std)


def _token_ids(case, seed):
    """[seqs, length] tokens, their frequencies falling with their rank, ranks spread over the table."""
    v, extra = case["vocab"], int(case["shifted"])
    cdf = torch.arange(v, device="cuda", dtype=torch.float64).add_(2.7).pow_(-case["skew"]).cumsum_(0)
    u = torch.rand(case["seqs"], case["length"] + extra, generator=_gen(seed, 1), device="cuda", dtype=torch.float64)
    ids = (torch.searchsorted(cdf, u * cdf[-1]).clamp_(max=v - 1) * 7919 + 13) % v
    if case["pad"]:  # the ends of the sequences are padding
        length = torch.randint(1, case["length"] + 1, (case["seqs"], 1), generator=_gen(seed, 2), device="cuda")
        ids[torch.arange(ids.shape[1], device="cuda")[None] >= length] = 0
    ids = ids if case["itype"] == "i64" else ids.to(torch.int32)
    return ids[:, :-1] if extra else ids


def _inputs(case, seed):
    s = dict(op=case["op"])
    if case["op"] in ("lookup", "grad"):
        s["ids"], s["scale"] = _token_ids(case, seed), math.sqrt(case["dim"])
        if case["op"] == "lookup":
            s["w"] = _randn((case["vocab"], case["dim"]), seed, 3, 0.02).to(TYPES[case["wtype"]])
            s["otype"] = TYPES[case["otype"]]
        else:
            s["dy"] = _randn((case["seqs"], case["length"], case["dim"]), seed, 4, 1e-3).to(TYPES[case["otype"]])
            s["dw"] = _randn((case["vocab"], case["dim"]), seed, 5, 1e-3).to(TYPES[case["wtype"]])
            s["pad"], s["tied"] = (0 if case["pad"] else None), case["tied"]
        return s
    sizes = _sizes(case)
    n, blocks = sum(sizes), [-(-k // BLOCK) for k in sizes]
    # a magnitude of its own for each tensor's gradient, over two decades
    std = torch.tensor([10.0 ** (-4 + 2 * ((k * 0.6180339887) % 1.0)) for k in range(len(sizes))], device="cuda")
    size = torch.tensor(sizes, device="cuda")
    g = _randn(n, seed, 6).mul_(torch.repeat_interleave(std, size, output_size=n))
    s.update(sizes=sizes, size=size, n=n, g=g.to(TYPES[case["gtype"]]), max_norm=1.0)
    if case["op"] == "norm":
        return s
    s["p"] = _randn(n, seed, 7, 0.02).to(TYPES[case["ptype"]])
    s["copy"] = torch.empty(n, device="cuda", dtype=torch.bfloat16) if case["copy"] else None
    # what the norm leaves on the device: the norm and the factor that the gradients are multiplied by
    s["clip"] = torch.tensor([2.7, 0.37], device="cuda") * (1 + 0.01 * _randn(1, seed, 8))
    s.update(t=case["t"], lr=case["lr"], seed=int(seed) % (1 << 40), bits=case["bits"])
    # weight decay for matrices and tables only
    s["decay"] = [case["decay"] if k >= 10_000 else 0.0 for k in sizes]
    if case["bits"] == 32:
        s["m"] = _randn(n, seed, 9, 0.3).mul_(g)
        s["v"] = _randn(n, seed, 10).square_().mul_(g).mul_(g)
    else:  # any states of the format: e4m3 values, and a power of two for each block
        nb = sum(blocks)
        s["m"] = _randn(n, seed, 9, 90.0).clamp_(-448, 448).to(torch.float8_e4m3fn)
        s["r"] = _randn(n, seed, 10, 90.0).abs_().clamp_(2.0 ** -9, 448).to(torch.float8_e4m3fn)
        e = torch.repeat_interleave(torch.log2(std).floor(), torch.tensor(blocks, device="cuda"), output_size=nb)
        s["m_scale"], s["r_scale"] = torch.exp2(e - 9), torch.exp2(e - 7)
    s["blocks"] = blocks
    return s


def _plan(s):
    """Where the plain 8-bit step finds each coordinate's block, its quad of random words and its word."""
    size, blocks = s["size"], torch.tensor(s["blocks"], device="cuda")
    n, nb, k = s["n"], sum(s["blocks"]), len(s["sizes"])
    quads = (size + 3) // 4
    nq = sum(-(-z // 4) for z in s["sizes"])
    first, first_quad, first_block = (c.cumsum(0) - c for c in (size, quads, blocks))
    which = torch.repeat_interleave(torch.arange(k, device="cuda"), size, output_size=n)
    j = torch.arange(n, device="cuda") - first[which]
    s["block"] = first_block[which] + j // BLOCK
    s["word"] = 4 * first_quad[which] + j
    s["quad_tensor"] = torch.repeat_interleave(torch.arange(k, device="cuda"), quads, output_size=nq)
    s["quad"] = torch.arange(nq, device="cuda") - first_quad[s["quad_tensor"]]
    s["nb"] = nb


def prepare(case, seed):
    s = _inputs(case, seed)
    s["own"] = own
    if not own:
        if case["op"] == "adamw":
            s["decays"] = torch.tensor(s["decay"], device="cuda")
            if case["bits"] == 8:
                _plan(s)
        return s
    import paper_2205_14473_gb300 as ea

    if case["op"] in ("lookup", "grad"):
        s["table"] = ea.Embedding(case["vocab"], case["dim"], max_tokens=s["ids"].numel(), scale=s["scale"],
                                  padding_idx=s.get("pad"))
        return s
    s["grads"] = ea.TensorList(s["g"].split(s["sizes"]))
    if case["op"] == "norm":
        s["norm"] = ea.GradNorm(s["sizes"], dtype=s["g"].dtype)
        return s
    states = {k: list(s[k].split(s["sizes"] if s[k].numel() == s["n"] and "scale" not in k else s["blocks"]))
              for k in ("m", "v", "r", "m_scale", "r_scale") if k in s}
    s["opt"] = ea.AdamW(list(s["p"].split(s["sizes"])), state_bits=case["bits"], betas=(BETA1, BETA2), eps=EPS,
                        weight_decay=s["decay"], grad_dtype=s["g"].dtype, states=states, seed=s["seed"], step=s["t"],
                        copies=None if s["copy"] is None else list(s["copy"].split(s["sizes"])))
    return s


# ------------------------------------------------------------------------------------ the plain forms

def _lookup(s):
    return (s["w"][s["ids"].reshape(-1).long()].float() * s["scale"]).to(s["otype"]).view(*s["ids"].shape, -1)


def _grad(s):
    ids, dim = s["ids"].reshape(-1).long(), s["dw"].shape[1]
    dy = s["dy"].reshape(-1, dim).float() * s["scale"]
    if s["pad"] is not None:
        dy = dy * (ids != s["pad"])[:, None]
    total = s["dw"].float() if s["tied"] else torch.zeros_like(s["dw"], dtype=torch.float32)
    if total is s["dw"]:
        return total.index_add_(0, ids, dy)
    s["dw"].copy_(total.index_add_(0, ids, dy))
    return s["dw"]


def _norm(s):
    norm = s["g"].float().square().sum().sqrt()
    return torch.stack([norm, (s["max_norm"] / norm).clamp(max=1.0)])


def _f32(x):
    return float(np.float32(x))


def _coefficients(s):
    """Step size, epsilon and decay rates of the step, the bias corrections folded into them."""
    t = s["t"] + 1
    root = math.sqrt(1 - _f32(BETA2) ** t)
    return s["lr"] * root / (1 - _f32(BETA1) ** t), _f32(EPS) * root


def _random(s):
    """Philox4x32-10 (Salmon et al., SC'11): four words for each quad of coordinates; key: the seed, counter:
    the quad, its tensor and the step."""
    mask, seed = 0xFFFFFFFF, s["seed"]
    c = [s["quad"] & mask, s["quad"] >> 32, s["quad_tensor"], torch.full_like(s["quad"], s["t"])]
    k0, k1 = seed & mask, (seed >> 32) & mask
    for _ in range(10):
        p0, p1 = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [((p1 >> 32) & mask) ^ c[1] ^ k0, p1 & mask, ((p0 >> 32) & mask) ^ c[3] ^ k1, p0 & mask]
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    return torch.stack(c, 1).reshape(-1)[s["word"]]


def _to_8_bits(s, x, random, codes, scale):
    """|x| in e4m3 steps of its block's power of two, rounded up with the probability of the rest."""
    most = torch.zeros(s["nb"], device="cuda").scatter_reduce_(0, s["block"], x, "amax")
    k = (((most.view(torch.int32) + 0x1FFFFF) >> 23) - 135).clamp(min=-126)
    y = x * ((127 - k) << 23).view(torch.float32)[s["block"]]
    normal = ((y.view(torch.int32) + (random << 4).to(torch.int32)) & -0x100000).view(torch.float32)
    small = torch.floor(y * 512 + random.float() * 2.0 ** -16) * 2.0 ** -9
    scale.copy_(((127 + k) << 23).view(torch.float32))
    return torch.where(y >= 2.0 ** -6, normal, small)


def _adamw(s):
    a, eps = _coefficients(s)
    rate = torch.repeat_interleave(s["decays"] * s["lr"], s["size"], output_size=s["n"])
    g = s["g"].float() * s["clip"][1]
    c1, c2 = _f32(1 - _f32(BETA1)), _f32(1 - _f32(BETA2))
    if s["bits"] == 32:
        m, v = s["m"].mul_(BETA1).add_(g * c1), s["v"].mul_(BETA2).add_(g * g * c2)
        root = v.sqrt()
    else:
        m = s["m"].float() * s["m_scale"][s["block"]] * BETA1 + g * c1
        r = s["r"].float() * s["r_scale"][s["block"]]
        v = r * r * BETA2 + g * g * c2
        root, random = v.sqrt(), _random(s)
        q = _to_8_bits(s, m.abs(), random & 0xFFFF, s["m"], s["m_scale"])
        s["m"].copy_(torch.copysign(q, m))
        q = _to_8_bits(s, root, random >> 16, s["r"], s["r_scale"])
        s["r"].copy_(torch.where(v > 0, q.clamp(min=2.0 ** -9), q))
    p = s["p"].float()
    new = p - (p * rate + m / (root + eps) * a)
    s["p"].copy_(new)
    if s["copy"] is not None:
        s["copy"].copy_(new)
    s["t"] += 1
    return {k: s[k] for k in ("p", "copy", "m", "v", "r", "m_scale", "r_scale") if s.get(k) is not None}


def run(state):
    s = state
    if not s["own"]:
        return {"lookup": _lookup, "grad": _grad, "norm": _norm, "adamw": _adamw}[s["op"]](s)
    if s["op"] == "lookup":
        return s["table"].lookup(s["ids"], s["w"], dtype=s["otype"])
    if s["op"] == "grad":
        return s["table"].grad(s["ids"], s["dy"], out=s["dw"], accumulate=s["tied"])
    if s["op"] == "norm":
        return s["norm"](s["grads"], max_norm=s["max_norm"])
    s["opt"].step(s["grads"], lr=s["lr"], clip=s["clip"])
    return {k: s[k] for k in ("p", "copy", "m", "v", "r", "m_scale", "r_scale") if s.get(k) is not None}


# -------------------------------------------------------------------------------- what a pass cannot do without

def _distinct(case):
    """Expected number of different tokens of a case (its padding counted as one more of them)."""
    p = (np.arange(case["vocab"]) + 2.7) ** -case["skew"]
    t = case["seqs"] * case["length"]
    return float(np.sum(-np.expm1(t * (0.5 if case["pad"] else 1.0) * np.log1p(-p / p.sum() * (1 - 1e-12))))) + case["pad"]


def work(case):
    if case["op"] in ("lookup", "grad"):
        t, dim, rows = case["seqs"] * case["length"], case["dim"], _distinct(case)
        ids = t * (8 if case["itype"] == "i64" else 4)
        w, o = SIZE[case["wtype"]], SIZE[case["otype"]]
        if case["op"] == "lookup":
            return {"bytes": ids + rows * dim * w + t * dim * o, "flops": t * dim}
        # padding takes no gradient: on average half of each sequence's rows need not be read
        t = t * (0.5 if case["pad"] else 1.0)
        return {"bytes": ids + t * dim * o + (2 * rows if case["tied"] else case["vocab"]) * dim * w, "flops": t * dim}
    n = sum(_sizes(case))
    if case["op"] == "norm":
        return {"bytes": n * SIZE[case["gtype"]] + 8, "flops": 2 * n}
    p, g, copy = SIZE[case["ptype"]], SIZE[case["gtype"]], 2 * case["copy"]
    if case["bits"] == 32:
        return {"bytes": n * (2 * p + g + copy + 16), "flops": 16 * n}
    return {"bytes": n * (2 * p + g + copy + 4) + 16 * sum(-(-k // BLOCK) for k in _sizes(case)), "flops": 30 * n}


# ------------------------------------------------------------------------------------ the same in 64 bits

def _exact_quantized(x, block, nb, draw):
    """(values, scale) of the states' format, in 64 bits: the scale of a block is the smallest power of two that
    brings its largest magnitude to 448 or less, and at least 2^-126."""
    top = torch.zeros(nb, dtype=torch.float64, device="cuda").scatter_reduce_(0, block, x.abs(), "amax")
    scale = torch.exp2(torch.ceil(torch.log2((top / 448).clamp(min=2.0 ** -126))))
    y = x.abs() / scale[block]
    step = torch.exp2(torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - 3)
    q = torch.floor(y / step + draw / 65536.0) * step
    return q, scale


def _exact_words(seed, t, which, j):
    """The 32 random bits of coordinate j of tensor `which` at step t."""
    def mulhilo(a, b):  # 32 x 32 bits by halves of b
        lo, hi = a * (b & 0xFFFF), a * (b >> 16)
        total = lo + ((hi & 0xFFFF) << 16)
        return (hi >> 16) + (total >> 32), total & 0xFFFFFFFF

    x0, x1 = (j // 4) % 2 ** 32, (j // 4) // 2 ** 32
    x2, x3 = torch.full_like(j, which), torch.full_like(j, t)
    key = [seed % 2 ** 32, seed // 2 ** 32 % 2 ** 32]
    for r in range(10):
        ka, kb = (key[0] + r * 0x9E3779B9) % 2 ** 32, (key[1] + r * 0xBB67AE85) % 2 ** 32
        h0, l0 = mulhilo(0xD2511F53, x0)
        h1, l1 = mulhilo(0xCD9E8D57, x2)
        x0, x1, x2, x3 = h1 ^ x1 ^ ka, l1, h0 ^ x3 ^ kb, l0
    return torch.stack([x0, x1, x2, x3]).gather(0, (j % 4)[None])[0]


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "lookup":
        return torch.nn.functional.embedding(s["ids"].long(), s["w"].double()) * s["scale"]
    if case["op"] == "grad":
        ids, dy = s["ids"].reshape(-1).long(), s["dy"].reshape(-1, case["dim"])
        order = torch.argsort(ids, stable=True)
        if s["pad"] is not None:
            order = order[ids[order] != s["pad"]]
        total = s["dw"].double() if s["tied"] else torch.zeros(s["dw"].shape, dtype=torch.float64, device="cuda")
        for part in order.split(1 << 15):
            total.index_add_(0, ids[part], dy[part].double(), alpha=s["scale"])
        return total
    if case["op"] == "norm":
        norm = math.sqrt(sum(float(part.double().square().sum()) for part in s["g"].split(1 << 26)))
        return torch.tensor([norm, min(1.0, s["max_norm"] / norm)], dtype=torch.float64)
    b1, b2, eps, t = _f32(BETA1), _f32(BETA2), _f32(EPS), case["t"] + 1
    factor = float(s["clip"][1])
    out = {k: [] for k in ("p", "copy", "m", "v", "r", "m_scale", "r_scale") if s.get(k) is not None}
    at = first = 0
    for i, size in enumerate(s["sizes"]):
        for lo in range(0, size, 1 << 26):  # whole blocks
            hi = min(size, lo + (1 << 26))
            part, nb = slice(at + lo, at + hi), -(-(hi - lo) // BLOCK)
            g, p = s["g"][part].double() * factor, s["p"][part].double()
            if case["bits"] == 32:
                m, v = s["m"][part].double(), s["v"][part].double()
            else:
                j = torch.arange(lo, hi, device="cuda")
                block = (j - lo) // BLOCK
                here = slice(first + lo // BLOCK, first + lo // BLOCK + nb)
                m = s["m"][part].double() * s["m_scale"][here].double()[block]
                v = (s["r"][part].double() * s["r_scale"][here].double()[block]) ** 2
            m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
            step = (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + eps)
            new = p - _f32(case["lr"]) * (step + _f32(s["decay"][i]) * p)
            out["p"].append(new)
            if "copy" in out:
                out["copy"].append(new)
            if case["bits"] == 32:
                out["m"].append(m)
                out["v"].append(v)
                continue
            words = _exact_words(s["seed"], case["t"], i, j)
            q, scale = _exact_quantized(m, block, nb, words % 65536)
            out["m"].append(torch.where(m < 0, -q, q))
            out["m_scale"].append(scale)
            q, scale = _exact_quantized(v.sqrt(), block, nb, words // 65536)
            out["r"].append(torch.where(v > 0, q.clamp(min=2.0 ** -9), q))
            out["r_scale"].append(scale)
        at, first = at + size, first + -(-size // BLOCK)
    return {k: torch.cat(v) for k, v in out.items()}
