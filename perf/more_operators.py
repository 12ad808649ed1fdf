"""Timing cases of the operators that distil a frozen teacher's answers into the
policy, each through its public entry point:

- ``pack``: tensors in 8-bit floating point (e4m3, one power of two for each block
  of 128 columns of a row, or of 128 x 128 for weights), and read again;
- ``linear``: y = x w^T as a frozen model runs it: x packed in the call, w packed
  once, the product of both;
- ``top``: the largest k of each row of logits with their columns, ties to the lowest
  column, and the row's log-sum-exp;
- ``distill``: the divergence of the student's distribution over the vocabulary
  from the teacher's top logits, and (``grad``) its gradients.

A case fixes every size; the seed given to ``prepare`` draws the values.
"""
import math

import torch

own = False

DEV = "cuda"
BLOCK = 128
TOP = 448.0  # the largest number of e4m3


def listed():
    return [
        # a few rows of odd width
        dict(name="pack_odd", kind="pack", rows=37, cols=1001, block_rows=1, dtype="f32"),
        # the residual stream of a 7B-class layer's trajectory
        dict(name="pack_7b", kind="pack", rows=137895, cols=3584, block_rows=1, dtype="bf16"),
        # a projection of the 7B-class block, when a frozen model is loaded
        dict(name="pack_weight", kind="pack", rows=18944, cols=3584, block_rows=128, dtype="bf16"),
        # one token through the 7B-class block's projection: latency and the weight's bytes
        dict(name="linear_token", kind="linear", rows=1, cols=3584, outs=18944, block_rows=128),
        # a few sequences' tokens through the small workload's projection
        dict(name="linear_tokens", kind="linear", rows=24, cols=2048, outs=5504, block_rows=128),
        # a ragged batch, widths that end inside a block, a scale for each row of w
        dict(name="linear_odd", kind="linear", rows=777, cols=2040, outs=5001, block_rows=1),
        # a chunk of rows through the 7B-class projection
        dict(name="linear_7b", kind="linear", rows=8192, cols=3584, outs=18944, block_rows=128),
        # one token's logits
        dict(name="top_token", kind="top", rows=1, vocab=151936, ld=151936, k=20, dtype="f32", scale=1.0),
        # the action rows of the 7B-class batch
        dict(name="top_7b", kind="top", rows=7680, vocab=151936, ld=151936, k=64, dtype="bf16", scale=0.5),
        # a few rows against a small vocabulary, the loss alone
        dict(name="distill_odd", kind="distill", rows=37, hidden=200, vocab=1001, k=5, grad=False, given=False),
        # the small workload's action rows
        dict(name="distill_small", kind="distill", rows=1024, hidden=2048, vocab=32000, k=32, grad=True, given=True),
        # the 7B-class batch's
        dict(name="distill_7b", kind="distill", rows=7680, hidden=3584, vocab=151936, k=64, grad=True, given=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["pack"] * 2 + ["linear"] * 4 + ["top"] * 3 + ["distill"] * 3)
    if kind == "pack":
        cols = _log(rng, 20, 19000)
        if rng.random() < 0.5:
            cols = max(16, cols // 16 * 16)
        return dict(kind=kind, rows=_log(rng, 1, min(137895, 400000000 // cols)), cols=cols,
                    block_rows=rng.choice([1, 1, 128]), dtype=rng.choice(["bf16", "bf16", "f32"]) if cols < 1500 else "bf16")
    if kind == "linear":
        cols = _log(rng, 16, 8192)
        outs = _log(rng, 16, min(18944, 60000000 // cols))
        if rng.random() < 0.5:
            cols, outs = max(16, cols // 16 * 16), max(16, outs // 16 * 16)
        return dict(kind=kind, rows=_log(rng, 1, 8192), cols=cols, outs=outs, block_rows=rng.choice([1, 128, 128]))
    if kind == "top":
        vocab = _log(rng, 100, 151936)
        return dict(kind=kind, rows=_log(rng, 1, 7680), vocab=vocab, ld=vocab + rng.choice([0, 0, rng.randint(1, 100)]),
                    k=_log(rng, 1, min(256, vocab)), dtype=rng.choice(["bf16", "f32"]) if vocab < 70000 else "bf16",
                    scale=rng.choice([1.0, 0.5, rng.uniform(0.2, 2.0)]))
    vocab = _log(rng, 300, 151936)
    return dict(kind=kind, rows=_log(rng, 1, 7680), hidden=8 * _log(rng, 8, 448), vocab=vocab, k=_log(rng, 1, 128),
                grad=rng.random() < 0.7, given=rng.random() < 0.5)


# -------------------------------------------------------------------- inputs

def _dt(c):
    return torch.bfloat16 if c.get("dtype", "bf16") == "bf16" else torch.float32


def _normal(gen, *shape, std=1.0, dt=torch.bfloat16):
    return (torch.randn(*shape, generator=gen, device=DEV) * std).to(dt)


def _activations(gen, rows, cols, dt):
    """Values as a residual stream has them: a few columns are much larger, a few rows are zero."""
    x = torch.randn(rows, cols, generator=gen, device=DEV)
    x *= torch.where(torch.rand(cols, generator=gen, device=DEV) < 0.01, 30.0, 1.0)
    if rows > 8:
        x[torch.rand(rows, generator=gen, device=DEV) < 0.02] = 0
    return x.to(dt)


def prepare(c, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    st = {"c": c}
    if c["kind"] == "pack":
        st["x"] = _activations(gen, c["rows"], c["cols"], _dt(c))
    elif c["kind"] == "linear":
        st["x"] = _activations(gen, c["rows"], c["cols"], torch.bfloat16)
        # rows of a weight differ in size
        w = torch.randn(c["outs"], c["cols"], generator=gen, device=DEV) / math.sqrt(c["cols"])
        w *= torch.exp(0.5 * torch.randn(c["outs"], 1, generator=gen, device=DEV))
        st["w"] = _pack(w, c["block_rows"])  # codes and exponent bytes, as a frozen model keeps them
    elif c["kind"] == "top":
        z = _normal(gen, c["rows"], c["ld"], std=2.5, dt=_dt(c))
        if c["vocab"] > 64:  # columns that the vocabulary was filled up with
            z[:, c["vocab"] - 3:] = -math.inf
        st["z"] = z[:, :c["vocab"]]
    else:
        rows, hidden, vocab, k = c["rows"], c["hidden"], c["vocab"], c["k"]
        more = rows + rows // 3 + 1  # the action rows are some of the batch's
        st["h"] = _normal(gen, more, hidden)
        st["w"] = _normal(gen, vocab, hidden, std=2.0 / math.sqrt(hidden))
        st["row_index"] = torch.randperm(more, generator=gen, device=DEV)[:rows].sort().values.int()
        # distinct columns: k of them at equal distances behind a random first one
        first = torch.randint(0, vocab, (rows, 1), generator=gen, device=DEV)
        st["ids"] = ((first + torch.arange(k, device=DEV) * (vocab // k)) % vocab).int()
        st["logits"] = torch.randn(rows, k, generator=gen, device=DEV).mul_(2.5).add_(6).sort(1, descending=True).values
        if k > 2:  # some teachers' answers are shorter
            short = torch.rand(rows, generator=gen, device=DEV) < 0.1
            st["ids"][short, k - k // 3:] = -1
        st["t_lse"] = torch.logsumexp(st["logits"], 1) + 0.3 * torch.rand(rows, generator=gen, device=DEV) if c["given"] else None
        weight = torch.rand(rows, generator=gen, device=DEV) + 0.5
        weight[torch.rand(rows, generator=gen, device=DEV) < 0.05] = 0
        st["weight"] = weight
    return st


# --------------------------------------------------------------- plain forms

def _two_to(e):
    """2^(e - 127) for e in 0 .. 254, from its bits (a library's power may be off by one place)."""
    return torch.where(e > 0, e << 23, torch.full_like(e, 1 << 22)).int().view(torch.float32)


def _pack(x, block_rows):
    """Codes [rows, cols up to 16] and exponent bytes [blocks of columns, blocks of rows up to 16]
    of x: the least power of two 2^s (s >= -127) with max|x| <= 448 2^s for each block."""
    rows, cols = x.shape
    p = torch.nn.functional.pad(x.float(), (0, -cols % BLOCK, 0, -rows % block_rows))
    b = p.view(p.shape[0] // block_rows, block_rows, -1, BLOCK)
    frac, e = torch.frexp(b.abs().amax((1, 3)))  # frac in [1/2, 1)
    s = torch.where(frac <= TOP / 512, e - 9, e - 8).int().clamp(min=-127)
    s = torch.where(frac == 0, torch.full_like(s, -127), s)
    code = (b * _two_to(127 - s)[:, None, :, None]).to(torch.float8_e4m3fn)
    code = code.view(p.shape)[:rows, :cols].view(torch.uint8)
    code = torch.nn.functional.pad(code, (0, -cols % 16))
    return code.contiguous(), torch.nn.functional.pad((s + 127).to(torch.uint8).t(), (0, -s.shape[0] % 16)).contiguous()


def _unpack(code, exp, rows, cols, block_rows):
    s = _two_to(exp.t().int()).repeat_interleave(block_rows, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :cols]
    return code[:, :cols].view(torch.float8_e4m3fn).float() * s


def _run_top(st):
    c = st["c"]
    z = st["z"].float()
    value, column = torch.sort(z, dim=1, descending=True, stable=True)
    y = z * c["scale"]
    top = y.amax(1, keepdim=True)
    lse = (top + torch.log(torch.exp(y - top).sum(1, keepdim=True)))[:, 0]
    return {"ids": column[:, :c["k"]].int(), "logits": value[:, :c["k"]].contiguous(), "lse": lse}


SCALE, TEACHER = 0.9, 0.8  # of the student's and the teacher's logits (temperatures)


def _run_distill(st):
    c = st["c"]
    h, w = st["h"][st["row_index"]].float(), st["w"].float()
    has = st["ids"] >= 0
    ids = torch.where(has, st["ids"], torch.zeros_like(st["ids"])).long()
    t = torch.where(has, st["logits"] * TEACHER, torch.full_like(st["logits"], -math.inf))
    if st["t_lse"] is None:
        top = t.amax(1, keepdim=True)
        norm = top + torch.log(torch.exp(t - top).sum(1, keepdim=True))
    else:
        norm = st["t_lse"][:, None]
    p = torch.exp(t - norm)
    z = (h @ w.t()) * SCALE
    top = z.amax(1, keepdim=True)
    lse = top + torch.log(torch.exp(z - top).sum(1, keepdim=True))
    term = p * (t - norm - torch.gather(z, 1, ids) + lse)
    loss = torch.where(p > 0, term, torch.zeros_like(p)).sum(1) * st["weight"]
    out = {"loss_tok": loss, "loss_sum": loss.sum(0, keepdim=True) / c["rows"], "lse": lse[:, 0]}
    if not c["grad"]:
        return out
    g = st["weight"][:, None] / c["rows"]
    dz = torch.exp(z - lse) * (g * p.sum(1, keepdim=True))
    dz.scatter_add_(1, ids, -g * p)
    out["dh"] = (dz @ w * SCALE).to(torch.bfloat16)
    out["dw"] = (dz.t() @ h * SCALE).to(torch.bfloat16)
    return out


def run(st):
    c = st["c"]
    if own:
        from paper_2607_11185_amd import seg as S
        if c["kind"] == "pack":
            return S.seg_fp8_unpack(S.seg_fp8_pack(st["x"], c["block_rows"]), st["x"].dtype)
        if c["kind"] == "linear":
            w = S.Fp8(*st["w"], c["cols"], c["block_rows"])
            return S.seg_fp8_gemm(S.seg_fp8_pack(st["x"]), w)
        if c["kind"] == "top":
            return S.seg_top_logits(st["z"], c["k"], c["scale"])
        cfg = S.DistillCfg(SCALE, TEACHER, 1.0 / c["rows"], c["grad"])
        out = S.seg_distill_loss(st["h"], st["row_index"], st["w"], st["ids"], st["logits"], cfg,
                                 t_lse=st["t_lse"], row_weight=st["weight"], dw_dtype=torch.bfloat16)
        return {n: v for n, v in out.items() if v is not None}
    if c["kind"] == "pack":
        return _unpack(*_pack(st["x"], c["block_rows"]), *st["x"].shape, c["block_rows"]).to(st["x"].dtype)
    if c["kind"] == "linear":
        x = _unpack(*_pack(st["x"], 1), *st["x"].shape, 1)
        return (x @ _unpack(*st["w"], c["outs"], c["cols"], c["block_rows"]).t()).to(torch.bfloat16)
    if c["kind"] == "top":
        return _run_top(st)
    return _run_distill(st)


def _packed_bytes(rows, cols, block_rows):
    return rows * cols + -(-rows // block_rows) * -(-cols // BLOCK)


def work(c):
    if c["kind"] == "pack":  # read, packed, read again, written
        e = 2 if c["dtype"] == "bf16" else 4
        return {"bytes": 2 * e * c["rows"] * c["cols"] + 2 * _packed_bytes(c["rows"], c["cols"], c["block_rows"]),
                "flops": 4 * c["rows"] * c["cols"]}
    if c["kind"] == "linear":
        rows, n, k = c["rows"], c["outs"], c["cols"]
        return {"bytes": 2 * rows * k + _packed_bytes(n, k, c["block_rows"]) + 2 * rows * n,
                "flops": 2.0 * rows * n * k}
    if c["kind"] == "top":
        e = 2 if c["dtype"] == "bf16" else 4
        return {"bytes": c["rows"] * (e * c["vocab"] + 8 * c["k"] + 4), "flops": 4 * c["rows"] * c["vocab"]}
    rows, h, v, k = c["rows"], c["hidden"], c["vocab"], c["k"]
    small = rows * (8 * k + 16)
    if not c["grad"]:
        return {"bytes": 2 * (rows * h + v * h) + small, "flops": 2.0 * rows * h * v}
    return {"bytes": 2 * (2 * rows * h + 2 * v * h) + small, "flops": 6.0 * rows * h * v}


# ------------------------------------------------------------ exact, 64 bits

def _exact_values(x, block_rows):
    """What 8 bits keep of x (64 bits), some blocks of rows at a time: the nearest of the numbers n 2^q
    with n < 16 and q the number's own exponent less 3, or that of the smallest normal number."""
    rows, cols = x.shape
    out = torch.empty(rows, cols, dtype=torch.float64, device=x.device)
    many = max(1, 4096 // block_rows) * block_rows
    wide = -(-cols // BLOCK) * BLOCK
    for at in range(0, rows, many):
        p = x[at:at + many].double()
        n = -(-len(p) // block_rows) * block_rows
        full = torch.zeros(n, wide, dtype=torch.float64, device=x.device)
        full[:len(p), :cols] = p
        full = full.view(-1, block_rows, wide // BLOCK, BLOCK)
        top = full.abs().amax((1, 3), keepdim=True)
        s = torch.ceil(torch.log2(top.clamp(min=2.0 ** -200) / TOP)).clamp(min=-127)
        unit = (s.long() + 1023 << 52).view(torch.float64)  # the power of two by its bits
        unit = torch.where(top > TOP * unit, unit * 2, unit)  # a logarithm rounded to the wrong side
        unit = torch.where((top <= TOP / 2 * unit) & (unit > 2.0 ** -127), unit / 2, unit)
        v = full / unit
        bits = v.abs().clamp(min=2.0 ** -6).view(torch.int64) >> 52  # exponent of each number
        step = (bits - 3 << 52).view(torch.float64)
        got = torch.round(v / step) * step * unit
        out[at:at + many] = got.view(n, wide)[:len(p), :cols]
    return out


def exact(c, seed):
    st = prepare(c, seed)
    if c["kind"] == "pack":
        return _exact_values(st["x"], c["block_rows"])
    if c["kind"] == "linear":
        code, exp = st["w"]
        number = torch.arange(256, device=DEV)  # what each code says
        e, f = number >> 3 & 15, (number & 7).double()
        value = torch.where(e > 0, (1 + f / 8) * (e + 1016 << 52).view(torch.float64), f * 2.0 ** -9)
        value = torch.where(number >= 128, -value, value)
        w = value[code[:, :c["cols"]].long()]
        at = torch.arange(c["outs"], device=DEV) // c["block_rows"]
        for b in range(-(-c["cols"] // BLOCK)):
            w[:, b * BLOCK:(b + 1) * BLOCK] *= (exp[b, at].long() + 896 << 52).view(torch.float64)[:, None]
        return _exact_values(st["x"], 1) @ w.t()
    if c["kind"] == "top":
        ids, logits, lse = [], [], []
        for z in st["z"].split(max(1, 200000000 // c["vocab"])):
            # one whole number for value and column: the value's bits in order, then the columns backwards
            bits = z.float().view(torch.int32).long()
            bits = torch.where(bits < 0, -(bits & 0x7fffffff), bits)
            back = c["vocab"] - 1 - torch.arange(c["vocab"], device=DEV)
            best = torch.topk((bits << 20) + back, c["k"], dim=1).values
            column = c["vocab"] - 1 - (best & (1 << 20) - 1)
            ids.append(column.int())
            logits.append(torch.gather(z, 1, column).double())
            lse.append(torch.logsumexp(z.double() * c["scale"], 1))
        return {"ids": torch.cat(ids), "logits": torch.cat(logits), "lse": torch.cat(lse)}
    rows, n = c["rows"], max(1, 200000000 // c["vocab"])
    w = st["w"].double()
    got = {n: [] for n in ("loss_tok", "lse", "dh")}
    dw = torch.zeros_like(w) if c["grad"] else None
    for at in range(0, rows, n):
        to = slice(at, at + n)
        h = st["h"][st["row_index"][to].long()].double()
        logq = torch.addmm(torch.zeros(1, dtype=torch.float64, device=DEV), h, w.t(), alpha=SCALE)
        lse = torch.logsumexp(logq, 1)
        logq -= lse[:, None]
        teacher = torch.zeros_like(logq)  # probabilities over the whole vocabulary
        t = st["logits"][to].double() * TEACHER
        r, j = torch.nonzero(st["ids"][to] >= 0, as_tuple=True)
        e = torch.zeros_like(t)
        e[r, j] = torch.exp(t[r, j] - (0 if st["t_lse"] is None else st["t_lse"][to].double()[r]))
        if st["t_lse"] is None:
            e /= e.sum(1, keepdim=True)
        teacher[r, st["ids"][to][r, j].long()] = e[r, j]
        kl = torch.special.xlogy(teacher, teacher) - teacher * logq
        weight = st["weight"][to].double()
        got["loss_tok"].append(kl.sum(1) * weight)
        got["lse"].append(lse)
        if c["grad"]:
            dz = torch.exp(logq) * teacher.sum(1, keepdim=True) - teacher
            dz *= weight[:, None] / rows
            got["dh"].append(SCALE * (dz @ w))
            dw += SCALE * (dz.t() @ h)
    out = {"loss_tok": torch.cat(got["loss_tok"]), "lse": torch.cat(got["lse"])}
    out["loss_sum"] = out["loss_tok"].sum(0, keepdim=True) / rows
    if c["grad"]:
        out["dh"], out["dw"] = torch.cat(got["dh"]), dw
    return out
