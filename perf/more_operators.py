"""The timed operators inside a residual block of a language model, between the lookup and the head.

A block normalises its input, runs a gated linear recurrence along each sequence, and adds what it made to the
input again, some of it dropped out; training takes each of the three back.  Every case is one call:

  layernorm   y = (x - mean) / sqrt(var + eps) * w + b, and each row's mean and 1 / sqrt(var + eps)
  layernorm_grad   the gradients of x (the residual's gradient added to it), w and b
  scan        h_t = f_t h_{t-1} + (1 - f_t) v_t, f = sigmoid(z), along every sequence, and its last state
  scan_grad   the gradients of z, v and the first state
  dropout     y = residual + x * kept / (1 - p), kept from a counter-based generator
  dropout_grad   dx = dy * kept / (1 - p), the same values kept
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5

# ---------------------------------------------------------------------------------------------- cases
# seqs sequences of length tokens, each a row of dim values.
# layernorm*: xtype of x, dx and the residual's gradient, ytype of y and dy, wtype of w, b and their gradients; plus:
#   dx has the residual's gradient added; sums: the gradients of w and b are added to what their buffers hold.
# scan*: xtype of z, v, h and their gradients; halves: z and v (and their gradients) are the halves of one product's
#   rows; state: there is a first state, and the last one (its gradient) is asked for (given); ragged: every sequence
#   has a length of its own; step: one token each of many sequences, the state updated in place.
# dropout*: xtype of x and dx, ytype of the residual, y and dy; p: of being dropped.


def _norm(name, op="layernorm", **kw):
    c = dict(op=op, seqs=1, length=1, dim=1600, xtype="bf16", ytype="bf16", wtype="f32")
    if op == "layernorm_grad":
        c.update(plus=True, sums=False)
    return _named(c, name, kw)


def _scan(name, op="scan", **kw):
    c = dict(op=op, seqs=16, length=1024, dim=1600, xtype="bf16", halves=True, state=False, ragged=False)
    if op == "scan":
        c["step"] = False
    return _named(c, name, kw)


def _drop(name, op="dropout", **kw):
    c = dict(op=op, seqs=16, length=1024, dim=1600, xtype="bf16", ytype="bf16", p=0.1)
    return _named(c, name, kw)


def _named(c, name, kw):
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one new token: the latency of a norm
        _norm("layernorm_one_row"),
        # a worker's batch of the GPT-2-XL-sized model
        _norm("layernorm_16k", seqs=16, length=1024),
        # the way back of that batch, with the gradient that passes the block by
        _norm("layernorm_grad_16k", "layernorm_grad", seqs=16, length=1024),
        # an odd width in 32 bits, the weight's gradient summed over several passes
        _norm("layernorm_grad_odd", "layernorm_grad", seqs=7, length=1003, dim=769, xtype="f32", ytype="f32", plus=False, sums=True),
        # generation: one token of each of 64 sequences
        _scan("scan_step_64", seqs=64, length=1, state=True, step=True),
        # the batch, z and v out of one product
        _scan("scan_16k"),
        # two long sequences
        _scan("scan_long", seqs=2, length=65536, dim=1024, state=True),
        # the way back of the batch
        _scan("scan_grad_16k", "scan_grad"),
        # sequences of uneven lengths in an odd layout, 32 bits, as a piece of longer ones
        _scan("scan_grad_ragged", "scan_grad", seqs=9, length=3001, dim=515, xtype="f32", halves=False, state=True, ragged=True),
        # one short sequence in 32 bits
        _drop("dropout_384", seqs=1, length=384, dim=768, xtype="f32", ytype="f32"),
        # the batch: what the block made, dropped out and added to the residual
        _drop("dropout_16k"),
        # the largest: the way back of many short texts, 32-bit gradients into 16-bit ones
        _drop("dropout_grad_256k", "dropout_grad", seqs=2048, length=127, dim=768, xtype="bf16", ytype="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["layernorm", "layernorm_grad", "layernorm_grad", "scan", "scan", "scan_grad", "scan_grad", "dropout", "dropout_grad"])
    dim = _log_int(rng, 32, 4096)
    dim = rng.choice([dim, -(-dim // 8) * 8, -(-dim // 64) * 64])
    same = rng.choice(["f32", "bf16", "bf16", "f16"])
    if op.startswith("scan"):
        most = 48_000_000 if op == "scan_grad" else 95_000_000
        length = _log_int(rng, 1, 65536)
        seqs = max(1, min(_log_int(rng, 1, 256), most // (dim * length)))
        length = min(length, most // (dim * seqs))
        step = op == "scan" and rng.random() < 0.2
        if step:
            length = 1
        kw = dict(seqs=seqs, length=length, dim=dim, xtype=same, halves=rng.random() < 0.5, state=step or rng.random() < 0.5,
                  ragged=not step and rng.random() < 0.4)
        return _scan("", op, **kw, **({"step": step} if op == "scan" else {}))
    length = _log_int(rng, 1, 2048)
    most = 70_000_000 if op == "layernorm_grad" else 95_000_000
    seqs = max(1, min(_log_int(rng, 1, 512), most // (dim * length)))
    mixed = rng.choice([("f32", "bf16"), ("f32", "f16")])
    if op.startswith("layernorm"):
        xtype, ytype = mixed if rng.random() < 0.3 else (same, same)
        kw = dict(seqs=seqs, length=length, dim=dim, xtype=xtype, ytype=ytype, wtype=rng.choice(["f32", "f32", ytype]))
        if op == "layernorm_grad":
            kw.update(plus=rng.random() < 0.5, sums=rng.random() < 0.4)
        return _norm("", op, **kw)
    xtype, ytype = mixed[::-1] if rng.random() < 0.3 else (same, same)
    return _drop("", op, seqs=seqs, length=length, dim=dim, xtype=xtype, ytype=ytype, p=rng.choice([0.05, 0.1, 0.1, 0.2, 0.5]))


# ---------------------------------------------------------------------------------- a case's inputs

def _randn(shape, seed, what, std=1.0, dtype=torch.float32):
    gen = torch.Generator(device="cuda").manual_seed(1 + 64 * (int(seed) % (1 << 40)) + what)
    return torch.randn(shape, generator=gen, device="cuda").mul_(std).to(dtype)


def _activations(case, seed, what):
    """Rows whose columns have offsets and a few much larger ones."""
    dim = case["dim"]
    x = _randn((case["seqs"], case["length"], dim), seed, what)
    spread = torch.exp(_randn((dim,), seed, what + 1, 0.4))
    spread[::97] *= 8.0
    return x.mul_(spread).add_(_randn((dim,), seed, what + 2, 0.3)).to(TYPES[case["xtype"]])


def _halves(case, seed, what, mean):
    """z and v: random, or where the case says so views of one tensor."""
    shape = (case["seqs"], case["length"], case["dim"])
    z, v = _randn(shape, seed, what, 1.5).add_(mean), _randn(shape, seed, what + 1)
    z, v = z.to(TYPES[case["xtype"]]), v.to(TYPES[case["xtype"]])
    if case["halves"]:
        return torch.cat([z, v], 2).split(case["dim"], 2)
    return z, v


def _inputs(case, seed):
    s = dict(op=case["op"])
    shape, dim = (case["seqs"], case["length"], case["dim"]), case["dim"]
    if case["op"].startswith("layernorm"):
        wt = TYPES[case["wtype"]]
        s["x"], s["ytype"] = _activations(case, seed, 1), TYPES[case["ytype"]]
        s["w"], s["b"] = _randn((dim,), seed, 5, 0.1).add_(1.0).to(wt), _randn((dim,), seed, 6, 0.1, wt)
        if case["op"] == "layernorm_grad":
            s["dy"] = _randn(shape, seed, 7, 0.01, s["ytype"])
            s["plus"] = _randn(shape, seed, 8, 0.01, s["x"].dtype) if case["plus"] else None
            s["dw"], s["db"], s["sums"] = _randn((dim,), seed, 9, 0.1, wt), _randn((dim,), seed, 10, 0.1, wt), case["sums"]
            # what the way there left: each row's mean and 1 / sqrt(var + eps)
            s["stats"] = torch.cat([_row_statistics(rows) for rows in s["x"].split(max(1, (1 << 25) // (dim * case["length"])))])
        return s
    if case["op"].startswith("scan"):
        s["z"], s["v"] = _halves(case, seed, 11, 1.5)
        s["step"] = case.get("step", False)
        s["initial"] = _randn((case["seqs"], dim), seed, 13) if case["state"] else None
        s["lengths"] = None
        if case["ragged"]:
            gen = torch.Generator(device="cuda").manual_seed(17 + 64 * (int(seed) % (1 << 40)))
            s["lengths"] = torch.randint(0, case["length"] + 1, (case["seqs"],), generator=gen, device="cuda")
        if case["op"] == "scan_grad":
            s["h"] = _states(s).to(s["z"].dtype)  # what the way there left
            s["dh"] = _randn(shape, seed, 14, 0.01, s["z"].dtype)
            s["d_final"] = _randn((case["seqs"], dim), seed, 15, 0.01) if case["state"] else None
            if case["halves"]:
                s["dz"], s["dv"] = torch.empty(*shape[:2], 2 * dim, device="cuda", dtype=s["z"].dtype).split(dim, 2)
            else:
                s["dz"], s["dv"] = torch.empty_like(s["z"]), torch.empty_like(s["v"])
        return s
    s.update(p=case["p"], seed=int(seed) % (1 << 40), counter=3 + int(seed) % 1000, xtype=TYPES[case["xtype"]], ytype=TYPES[case["ytype"]])
    if case["op"] == "dropout":
        s["x"], s["residual"] = _randn(shape, seed, 17, 1.0, s["xtype"]), _randn(shape, seed, 18, 2.0, s["ytype"])
    else:
        s["dy"] = _randn(shape, seed, 19, 0.01, s["ytype"])
    return s


def _row_statistics(x):
    x = x.double()
    mean = x.mean(-1)
    return torch.stack([mean, ((x - mean[..., None]).square().mean(-1) + EPS).rsqrt()], -1).float()


def prepare(case, seed):
    s = _inputs(case, seed)
    s["own"] = own
    if own:
        import paper_2205_14473_gb300 as ea

        if case["op"].startswith("layernorm"):
            s["norm"] = ea.LayerNorm(case["dim"], max_rows=case["seqs"] * case["length"], eps=EPS)
        elif case["op"].startswith("scan"):
            s["scan"] = ea.GatedScan(case["dim"])
        else:
            s["drop"] = ea.Dropout(case["p"], seed=s["seed"])
    return s


# ------------------------------------------------------------------------------------ the plain forms

def _layernorm(s):
    x = s["x"].float()
    mean = x.mean(-1, keepdim=True)
    x = x - mean
    rstd = 1.0 / (x.square().mean(-1, keepdim=True) + EPS).sqrt()
    return {"y": (x * rstd * s["w"].float() + s["b"].float()).to(s["ytype"]), "stats": torch.cat([mean, rstd], -1)}


def _layernorm_grad(s):
    dy, rstd = s["dy"].float(), s["stats"][..., 1:]
    xhat = (s["x"].float() - s["stats"][..., :1]) * rstd
    wdy = dy * s["w"].float()
    dx = (wdy - wdy.mean(-1, keepdim=True) - xhat * (wdy * xhat).mean(-1, keepdim=True)) * rstd
    if s["plus"] is not None:
        dx = dx + s["plus"].float()
    dw, db = (dy * xhat).sum((0, 1)), dy.sum((0, 1))
    if s["sums"]:
        dw, db = s["dw"].float() + dw, s["db"].float() + db
    s["dw"].copy_(dw)
    s["db"].copy_(db)
    return {"dx": dx.to(s["x"].dtype), "dw": s["dw"], "db": s["db"]}


def _recur(f, u):
    """x_t = f_t x_{t-1} + u_t along dimension 1, x before the first row 0: each pass joins every row with the rows that
    the one before it did not reach, twice as far back as the last."""
    reach, length = 1, f.shape[1]
    while reach < length:
        u = torch.cat([u[:, :reach], u[:, reach:] + f[:, reach:] * u[:, :-reach]], 1)
        f = torch.cat([f[:, :reach], f[:, reach:] * f[:, :-reach]], 1)
        reach *= 2
    return u


def _behind(s):
    """Which rows lie behind their sequence's end, or None."""
    if s["lengths"] is None:
        return None
    return (torch.arange(s["z"].shape[1], device="cuda") >= s["lengths"][:, None])[..., None]


def _states(s):
    """The states of every row in 32 bits; those behind a sequence's end zero."""
    f, behind = torch.sigmoid(s["z"].float()), _behind(s)
    u = (1.0 - f) * s["v"].float()
    if behind is not None:
        f, u = f.masked_fill(behind, 1.0), u.masked_fill(behind, 0.0)
    if s["initial"] is not None:
        u[:, 0] += f[:, 0] * s["initial"]
    h = _recur(f, u)
    s["last"] = h[:, -1].clone()
    return h if behind is None else h.masked_fill(behind, 0.0)


def _scan_plain(s):
    h = _states(s).to(s["z"].dtype)
    if s["step"]:
        s["initial"].copy_(s["last"])
        return {"h": h[:, 0], "state": s["initial"]}
    return {"h": h, "final": s["last"] if s["initial"] is not None else None}


def _scan_grad(s):
    f, behind, dh, h = torch.sigmoid(s["z"].float()), _behind(s), s["dh"].float(), s["h"].float()
    keep = f
    if behind is not None:
        keep, dh = f.masked_fill(behind, 1.0), dh.masked_fill(behind, 0.0)
    if s["d_final"] is not None:
        dh = torch.cat([dh[:, :-1], dh[:, -1:] + s["d_final"][:, None]], 1)
    # from the last row to the first: each row's gradient and the next one's times that one's f
    later = torch.cat([torch.zeros_like(keep[:, :1]), keep[:, 1:].flip(1)], 1)
    g = _recur(later, dh.flip(1)).flip(1)
    first = torch.zeros_like(h[:, 0]) if s["initial"] is None else s["initial"]
    before = torch.cat([first[:, None], h[:, :-1]], 1)
    d_initial = keep[:, 0] * g[:, 0]
    if behind is not None:
        g = g.masked_fill(behind, 0.0)
    s["dv"].copy_((1.0 - f) * g)
    s["dz"].copy_(f * (1.0 - f) * g * (before - s["v"].float()))
    return {"dz": s["dz"], "dv": s["dv"], "d_initial": d_initial if s["initial"] is not None else None}


def _kept(n, seed, counter, p):
    """Element j's half word j mod 8 of Philox4x32-10 (Salmon et al., SC'11) at the counter (j / 8, counter) under the key
    seed is at least 65536 p, rounded."""
    mask, blocks = 0xFFFFFFFF, torch.arange(-(-n // 8), device="cuda")
    c = [blocks & mask, blocks >> 32, torch.full_like(blocks, counter & mask), torch.full_like(blocks, counter >> 32)]
    k0, k1 = seed & mask, (seed >> 32) & mask
    for _ in range(10):
        p0, p1 = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [((p1 >> 32) & mask) ^ c[1] ^ k0, p1 & mask, ((p0 >> 32) & mask) ^ c[3] ^ k1, p0 & mask]
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    words = torch.stack(c, 1)
    return torch.stack([words & 0xFFFF, words >> 16], 2).reshape(-1)[:n] >= round(65536 * p)


def _dropout(s):
    x = s["x"] if s["op"] == "dropout" else s["dy"]
    kept = _kept(x.numel(), s["seed"], s["counter"], s["p"]).view(x.shape)
    y = torch.where(kept, x.float() * (65536.0 / (65536 - round(65536 * s["p"]))), 0.0)
    return (y + s["residual"].float()).to(s["ytype"]) if s["op"] == "dropout" else y.to(s["xtype"])


def run(state):
    s = state
    if not s["own"]:
        plain = {"layernorm": _layernorm, "layernorm_grad": _layernorm_grad, "scan": _scan_plain, "scan_grad": _scan_grad}
        return plain.get(s["op"], _dropout)(s)
    if s["op"] == "layernorm":
        y, stats = s["norm"].forward(s["x"], s["w"], s["b"], dtype=s["ytype"])
        return {"y": y, "stats": stats}
    if s["op"] == "layernorm_grad":
        dx, dw, db = s["norm"].grad(s["dy"], s["x"], s["stats"], s["w"], add=s["plus"], dw=s["dw"], db=s["db"], accumulate=s["sums"])
        return {"dx": dx, "dw": dw, "db": db}
    if s["op"] == "scan":
        if s["step"]:
            h = s["scan"].step(s["z"][:, 0], s["v"][:, 0], s["initial"])
            return {"h": h, "state": s["initial"]}
        h, final = s["scan"].forward(s["z"], s["v"], initial=s["initial"], lengths=s["lengths"], final=s["initial"] is not None)
        return {"h": h, "final": final}
    if s["op"] == "scan_grad":
        dz, dv, d_initial = s["scan"].grad(s["dh"], s["z"], s["v"], s["h"], initial=s["initial"], lengths=s["lengths"],
                                           d_final=s["d_final"], dz=s["dz"], dv=s["dv"], d_initial=s["initial"] is not None)
        return {"dz": dz, "dv": dv, "d_initial": d_initial}
    if s["op"] == "dropout":
        return s["drop"](s["x"], s["counter"], residual=s["residual"])
    return s["drop"].grad(s["dy"], s["counter"], dtype=s["xtype"])


# -------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    rows, dim = case["seqs"] * case["length"], case["dim"]
    n, x = rows * dim, SIZE[case["xtype"]]
    if case["op"] == "layernorm":
        return {"bytes": n * (x + SIZE[case["ytype"]]) + 8 * rows + 2 * dim * SIZE[case["wtype"]], "flops": 8 * n}
    if case["op"] == "layernorm_grad":
        return {"bytes": n * (SIZE[case["ytype"]] + (2 + case["plus"]) * x) + 8 * rows + (3 + 2 * case["sums"]) * dim * SIZE[case["wtype"]],
                "flops": 14 * n}
    if case["op"].startswith("scan"):
        # on average half of a ragged batch need not be read
        read = 0.5 if case["ragged"] else 1.0
        states = 8 * case["seqs"] * dim if case["state"] else 0
        if case["op"] == "scan":
            return {"bytes": n * x * (2 * read + 1) + states, "flops": 8 * n * read}
        return {"bytes": n * x * (4 * read + 2) + 2 * states, "flops": 14 * n * read}
    y = SIZE[case["ytype"]]
    return {"bytes": n * (x + (2 * y if case["op"] == "dropout" else y)), "flops": 12 * n}


# ------------------------------------------------------------------------------------ the same in 64 bits

def _exact_norm(s):
    x = s["x"].to(torch.float64)
    centre = x.sum(-1, keepdim=True) / x.shape[-1]
    spread = torch.sqrt(((x - centre) ** 2).sum(-1, keepdim=True) / x.shape[-1] + EPS)
    if s["op"] == "layernorm":
        return {"y": (x - centre) / spread * s["w"] + s["b"], "stats": torch.cat([centre, 1 / spread], -1)}
    # of the statistics that are given
    r = s["stats"][..., 1].double().unsqueeze(-1)
    t, dy = (x - s["stats"][..., 0].double().unsqueeze(-1)) * r, s["dy"].double()
    q, n = s["w"].double() * dy, x.shape[-1]
    dx = r * (q - q.sum(-1, keepdim=True) / n - t * ((q * t).sum(-1, keepdim=True) / n))
    if s["plus"] is not None:
        dx += s["plus"]
    dw, db = torch.einsum("abc,abc->c", dy, t), torch.einsum("abc->c", dy)
    return {"dx": dx, "dw": dw + s["dw"] if s["sums"] else dw, "db": db + s["db"] if s["sums"] else db}


def _exact_scan(s):
    """Row after row, forward or backward, a sequence's state staying as it is behind its end."""
    seqs, length, dim = s["z"].shape
    ends = [length] * seqs if s["lengths"] is None else s["lengths"].tolist()
    zero = torch.zeros(seqs, dim, dtype=torch.float64, device="cuda")
    inside = (torch.arange(length)[None, :, None] < torch.tensor(ends)[:, None, None]).double().cuda()
    f = 1 / (1 + torch.exp(-s["z"].double()))
    stay = f * inside + (1 - inside)
    if s["op"] == "scan":
        state, new = zero if s["initial"] is None else s["initial"].double(), s["v"].double() / (1 + torch.exp(s["z"].double())) * inside
        h = torch.empty_like(f)
        for t in range(length):
            state = torch.addcmul(new[:, t], stay[:, t], state, out=h[:, t])
        last = state.clone()
        if s["step"]:
            return {"h": h[:, 0], "state": last}
        return {"h": h.mul_(inside), "final": last if s["initial"] is not None else None}
    g = torch.empty_like(f)
    late, dh = (zero if s["d_final"] is None else s["d_final"].double()), s["dh"].double() * inside
    for t in reversed(range(length)):
        late = dh[:, t] + (late if t == length - 1 else stay[:, t + 1] * late)
        g[:, t] = late
    g_in = g * inside
    before = torch.empty_like(f)
    before[:, 0] = zero if s["initial"] is None else s["initial"].double()
    before[:, 1:] = s["h"][:, :-1]
    shut = 1 / (1 + torch.exp(s["z"].double()))
    return {"dz": g_in * f * shut * (before - s["v"].double()), "dv": g_in * shut,
            "d_initial": stay[:, 0] * g[:, 0] if s["initial"] is not None else None}


def _exact_mask(n, seed, counter):
    """The 16 random bits of each of n elements."""
    def mulhilo(a, b):  # 32 x 32 bits by halves of b
        lo, hi = a * (b & 0xFFFF), a * (b >> 16)
        total = lo + ((hi & 0xFFFF) << 16)
        return (hi >> 16) + (total >> 32), total & 0xFFFFFFFF

    j = torch.arange((n + 7) // 8, device="cuda")
    x0, x1 = j % 2 ** 32, j // 2 ** 32
    x2, x3 = torch.full_like(j, counter % 2 ** 32), torch.full_like(j, counter // 2 ** 32)
    key = [seed % 2 ** 32, seed // 2 ** 32 % 2 ** 32]
    for r in range(10):
        ka, kb = (key[0] + r * 0x9E3779B9) % 2 ** 32, (key[1] + r * 0xBB67AE85) % 2 ** 32
        h0, l0 = mulhilo(0xD2511F53, x0)
        h1, l1 = mulhilo(0xCD9E8D57, x2)
        x0, x1, x2, x3 = h1 ^ x1 ^ ka, l1, h0 ^ x3 ^ kb, l0
    bits = torch.empty(j.numel(), 8, dtype=torch.int32, device="cuda")
    for i, x in enumerate((x0, x1, x2, x3)):
        bits[:, 2 * i], bits[:, 2 * i + 1] = x % 65536, x // 65536
    return bits.view(-1)[:n]


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"].startswith("layernorm"):
        return _exact_norm(s)
    if case["op"].startswith("scan"):
        return _exact_scan(s)
    x = s["x"] if case["op"] == "dropout" else s["dy"]
    limit = round(65536 * case["p"])
    kept = (_exact_mask(x.numel(), s["seed"], s["counter"]) >= limit).view(x.shape)
    y = x.double() / (1 - limit / 65536) * kept
    return y + s["residual"] if case["op"] == "dropout" else y
