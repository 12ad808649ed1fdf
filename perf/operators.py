"""Timing cases of the operators that the decoder layer of a vision-language
model is trained with, each through its public entry point:

- ``pos``: the time, height and width position of every row of a packed layout;
- ``rope``: rotation of q and k by such positions, and (``inverse``) of their
  gradients back;
- ``act``: activations kept in 8 bits and read again (blocks of 32 columns with
  a power of two each);
- ``glu``: the gated feed-forward block silu(x Wg^T) * (x Wu^T), with its gate
  and up values kept in 8 bits (``keep``), and (``grad``) its backward from the
  kept values.

A case fixes every size; the seed given to ``prepare`` draws the values.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
BLOCK = 32


def listed():
    return [
        # the positions of the 7B-class batch: 8 trajectories of 30 turns, 69 x 39 merged
        # patches a screenshot, segments of 5 turns; every batch needs them once
        dict(name="pos_7b", kind="pos", traj=8, turns=30, prompt=512, text_lo=150, text_hi=400, gt=1, gh=39,
             gw=69, window=3, seg_steps=5, buffer=0, spans=0),
        # the long workload's 50-turn trajectories in padded buffers, with clips of four frames
        dict(name="pos_long_clips", kind="pos", traj=16, turns=40, prompt=512, text_lo=100, text_hi=600, gt=4,
             gh=16, gw=64, window=5, seg_steps=8, buffer=65536, spans=1),
        # one token on its way into a cache: latency
        dict(name="rope_token", kind="rope", rows=1, hq=28, hkv=4, d=128, s0=16, s1=24, s2=24, dtype="bf16",
             inverse=False, fused=True, far=40000),
        # a trajectory's q and k, read from the rows of one projection output
        dict(name="rope_7b", kind="rope", rows=137895, hq=28, hkv=4, d=128, s0=16, s1=24, s2=24, dtype="bf16",
             inverse=False, fused=True, far=25000),
        # gradients of a small batch in fp32, 64 columns a head, far positions
        dict(name="rope_grad_f32", kind="rope", rows=10007, hq=12, hkv=4, d=64, s0=8, s1=12, s2=12,
             dtype="f32", inverse=True, fused=False, far=1000000),
        # a few rows of odd width
        dict(name="act_odd", kind="act", rows=37, cols=1001, dtype="f32"),
        # the residual stream of a 7B-class layer's trajectory
        dict(name="act_7b", kind="act", rows=137895, cols=3584, dtype="bf16"),
        # four tokens through the 7B-class block: the weights' bytes count
        dict(name="glu_tokens", kind="glu", rows=4, hidden=3584, inter=18944, keep=False, grad=False),
        # the small workload's width, a ragged number of rows, values kept
        dict(name="glu_small", kind="glu", rows=1500, hidden=2048, inter=5504, keep=True, grad=False),
        # a chunk of rows of the 7B-class layer, values kept
        dict(name="glu_7b", kind="glu", rows=8192, hidden=3584, inter=18944, keep=True, grad=False),
        # their backwards
        dict(name="glu_small_grad", kind="glu", rows=1500, hidden=2048, inter=5504, keep=True, grad=True),
        dict(name="glu_7b_grad", kind="glu", rows=8192, hidden=3584, inter=18944, keep=True, grad=True),
    ]


HEADS = [(4, 1, 64), (12, 4, 64), (16, 2, 128), (28, 4, 128), (7, 1, 128), (6, 6, 128), (8, 8, 64)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["pos"] * 2 + ["rope"] * 3 + ["act"] * 3 + ["glu"] * 5)
    if kind == "pos":
        lo, h = rng.randint(8, 200), rng.randint(2, 40)
        c = dict(kind=kind, traj=rng.randint(1, 12), turns=rng.randint(6, 40), prompt=rng.choice([1, rng.randint(1, 900)]),
                 text_lo=lo, text_hi=lo + rng.randint(0, 400), gt=rng.choice([1, 1, rng.randint(2, 6)]), gh=h,
                 gw=h + rng.randint(1, 32), window=rng.randint(1, 6), seg_steps=rng.randint(1, 10), buffer=0,
                 spans=rng.randrange(1 << 20))
        while (sizes := _segment_rows(c)) and sum(sizes) > 2000000:
            c["traj"], c["turns"], c["gt"] = max(1, c["traj"] - 1), max(6, c["turns"] * 4 // 5), 1
        if rng.random() < 0.3:
            c["buffer"] = max(sizes) + rng.randint(0, 3000)
        return c
    if kind == "rope":
        hq, hkv, d = rng.choice(HEADS)
        s0 = rng.randint(0, d // 4)
        s1 = rng.randint(0, d // 2 - s0)
        return dict(kind=kind, rows=_log(rng, 1, 130000), hq=hq, hkv=hkv, d=d, s0=s0, s1=s1, s2=d // 2 - s0 - s1,
                    dtype=rng.choice(["bf16", "bf16", "f32"]) if hq * d < 2048 else "bf16",
                    inverse=rng.random() < 0.5, fused=rng.random() < 0.5, far=_log(rng, 1000, 1000000))
    if kind == "act":
        cols = _log(rng, 20, 19000)
        if rng.random() < 0.6:
            cols = max(8, cols // 8 * 8)
        return dict(kind=kind, rows=_log(rng, 1, min(130000, 400000000 // cols)), cols=cols,
                    dtype=rng.choice(["bf16", "bf16", "f32"]) if cols < 1500 else "bf16")
    hidden = 8 * _log(rng, 16, 448)
    grad = rng.random() < 0.4
    return dict(kind=kind, rows=_log(rng, 1, 8192), hidden=hidden,
                inter=min(18944, 8 * int(hidden * rng.uniform(2.0, 5.3) / 8)), keep=grad or rng.random() < 0.6, grad=grad)


# -------------------------------------------------------------------- inputs

def _dt(c):
    return torch.bfloat16 if c.get("dtype", "bf16") == "bf16" else torch.float32


def _spans(c):
    """Text lengths of every turn (part of the case, not of the seed)."""
    r = np.random.default_rng([c["spans"], 77])
    return r.integers(c["text_lo"], c["text_hi"] + 1, size=(c["traj"], c["turns"])).astype(np.int32)


def _runs(c):
    """Every token run of the packed segments: first row, rows, step (-1: text or prompt) and
    segment; and the packed rows.  Segment [a, b): the prompt, then for each turn j < b its screenshot
    if j > a - window, and its text."""
    text, img = _spans(c), c["gt"] * c["gh"] * c["gw"]
    first, rows, step, seg = [], [], [], []
    at, fill, nbuf, n = 0, 0, 0, 0
    for t in range(c["traj"]):
        for a in range(1, c["turns"] + 1, c["seg_steps"]):
            b = min(a + c["seg_steps"], c["turns"] + 1)
            here = [(c["prompt"], -1)]
            for j in range(1, b):
                if j > a - c["window"]:
                    here.append((img, t * c["turns"] + j - 1))
                here.append((int(text[t, j - 1]), -1))
            size = sum(x for x, _ in here)
            if c["buffer"]:
                if nbuf == 0 or fill + size > c["buffer"]:
                    at, fill, nbuf = nbuf * c["buffer"], 0, nbuf + 1
                fill += size
            for x, s in here:
                first.append(at)
                rows.append(x)
                step.append(s)
                seg.append(n)
                at += x
            n += 1
    return first, rows, step, seg, nbuf * c["buffer"] if c["buffer"] else at


def _segment_rows(c):
    rows = {}
    for x, q in zip(*(_runs(c)[k] for k in (1, 3))):
        rows[q] = rows.get(q, 0) + x
    return list(rows.values())


def _grids(c, seed):
    """(frames, height, width, time step) of every turn's screenshot: its patches are the case's, their
    arrangement and the time step are drawn."""
    r = np.random.default_rng([seed, 78])
    n = c["traj"] * c["turns"]
    g = np.empty((n, 4), np.int32)
    g[:, 0] = c["gt"]
    turn = r.random(n) < 0.5
    g[:, 1] = np.where(turn, c["gw"], c["gh"])
    g[:, 2] = np.where(turn, c["gh"], c["gw"])
    g[:, 3] = r.integers(1, 5, n)
    return g


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
    if c["kind"] == "pos":
        grid = _grids(c, seed)
        if own:
            from paper_2607_11185_amd import seg as S
            from paper_2607_11185_amd import workload as WL
            n, img = c["traj"] * c["turns"], c["gt"] * c["gh"] * c["gw"]
            sp = WL.explicit_spans([c["turns"]] * c["traj"], [c["prompt"]] * c["traj"], [img] * n, _spans(c).reshape(-1), [1] * n)
            st["problem"] = S.Problem.from_spans(sp, c["window"], c["seg_steps"], 0, c["buffer"])
            st["layout"] = S.seg_build_layout(st["problem"], device=DEV)
            st["grid"] = grid
            return st
        first, rows, step, seg, total = _runs(c)
        st["first"], st["rows"], st["seg"] = (torch.tensor(v, device=DEV) for v in (first, rows, seg))
        st["total"] = total
        step = np.array(step)
        g = np.where((step >= 0)[:, None], grid[np.maximum(step, 0)], 0)  # zeros: a run of text
        st["grid"] = torch.tensor(g.astype(np.int64), device=DEV)
    elif c["kind"] == "rope":
        rows, hq, hkv, d = c["rows"], c["hq"], c["hkv"], c["d"]
        if c["fused"]:  # rows of [q heads | k heads | v heads]
            x = _normal(gen, rows, hq + 2 * hkv, d, dt=_dt(c))
            st["q"], st["k"] = x[:, :hq], x[:, hq:hq + hkv]
        else:
            st["q"], st["k"] = _normal(gen, rows, hq, d, dt=_dt(c)), _normal(gen, rows, hkv, d, dt=_dt(c))
        pos = torch.randint(0, c["far"], (3, rows), generator=gen, device=DEV, dtype=torch.int32)
        if rows > 8:
            pos[:, torch.rand(rows, generator=gen, device=DEV) < 0.02] = -1
        st["pos"] = pos
    elif c["kind"] == "act":
        st["x"] = _activations(gen, c["rows"], c["cols"], _dt(c))
    else:
        rows, h, i = c["rows"], c["hidden"], c["inter"]
        st["x"] = _normal(gen, rows, h)
        st["wg"], st["wu"] = _normal(gen, i, h, std=1.5 / math.sqrt(h)), _normal(gen, i, h, std=1.0 / math.sqrt(h))
        if c["grad"]:
            st["dm"] = _normal(gen, rows, i, std=0.05)
            # codes and exponent bytes of the gate and up values of these inputs
            st["kept"] = [_pack((st["x"] @ st[w].t()).float()) for w in ("wg", "wu")]
    return st


# --------------------------------------------------------------- plain forms

def _two_to(e):
    """2^(e - 127) for e in 0 .. 254, from its bits (a library's power may be off by one place)."""
    return torch.where(e > 0, e << 23, torch.full_like(e, 1 << 22)).int().view(torch.float32)


def _pack(x):
    """Codes and exponent bytes of x: the least power of two 2^s (s >= -127) with max|x| <= 127 2^s
    for each block of 32 columns of a row."""
    rows, cols = x.shape
    b = torch.nn.functional.pad(x, (0, -cols % BLOCK)).view(rows, -1, BLOCK)
    frac, e = torch.frexp(b.abs().amax(-1))  # frac in [1/2, 1)
    s = torch.where(frac <= 127 / 128, e - 7, e - 6).int().clamp(min=-127)
    s = torch.where(frac == 0, torch.full_like(s, -127), s)
    code = torch.round(b * _two_to(127 - s)[..., None])
    return code.view(rows, -1)[:, :cols].to(torch.int8).contiguous(), (s + 127).to(torch.uint8)


def _unpack(code, exp, dt):
    s = _two_to(exp.int()).repeat_interleave(BLOCK, 1)[:, :code.shape[1]]
    return (code.float() * s).to(dt)


def _run_pos(st):
    first, rows, grid = st["first"], st["rows"], st["grid"]
    t, h, w, e = grid.unbind(1)
    is_text = h == 0
    adv = torch.where(is_text, rows, torch.maximum(torch.maximum(h, w), e * (t - 1) + 1))
    before = torch.cumsum(adv, 0) - adv
    opens = torch.cat([torch.ones_like(st["seg"][:1], dtype=torch.bool), st["seg"][1:] != st["seg"][:-1]])
    start = before - before[opens][st["seg"]]
    run = torch.repeat_interleave(torch.arange(len(rows), device=DEV), rows)
    at = torch.arange(len(run), device=DEV) - (torch.cumsum(rows, 0) - rows)[run]
    hw, w1 = (h * w).clamp(min=1)[run], w.clamp(min=1)[run]
    text, n = is_text[run], start[run]
    pos = torch.full((3, st["total"]), -1, dtype=torch.int32, device=DEV)
    row = first[run] + at
    for axis, off in enumerate((at // hw * e[run], at // w1 % h.clamp(min=1)[run], at % w1)):
        pos[axis, row] = (n + torch.where(text, at, off)).int()
    return pos


def _run_rope(st):
    c, pos = st["c"], st["pos"]
    half = c["d"] // 2
    axis = torch.repeat_interleave(torch.arange(3, device=DEV), torch.tensor([c["s0"], c["s1"], c["s2"]], device=DEV))
    freq = torch.exp2(torch.arange(half, device=DEV, dtype=torch.float64) * (-2.0 / c["d"] * math.log2(1e6)))
    angle = pos[axis].t().double() * freq
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if c["inverse"]:
        sin = -sin
    pad = (pos < 0).any(0)[:, None, None]
    out = []
    for x in (st["q"], st["k"]):
        a, b = x[..., :half].float(), x[..., half:].float()
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(x.dtype)
        out.append(torch.where(pad, torch.zeros_like(y) if c["inverse"] else x, y))
    return out


def _run_glu(st):
    c = st["c"]
    x, wg, wu = st["x"].float(), st["wg"].float(), st["wu"].float()
    if not c["grad"]:
        g, u = x @ wg.t(), x @ wu.t()
        out = {"m": (g * torch.sigmoid(g) * u).to(torch.bfloat16)}
        if c["keep"]:
            out["g"], out["u"] = _unpack(*_pack(g), torch.bfloat16), _unpack(*_pack(u), torch.bfloat16)
        return out
    dm = st["dm"].float()
    g, u = (_unpack(*kept, torch.float32) for kept in st["kept"])
    s = torch.sigmoid(g)
    dg, du = dm * u * s * (1 + g * (1 - s)), dm * g * s
    got = {"m": g * s * u, "dx": dg @ wg + du @ wu, "dwg": dg.t() @ x, "dwu": du.t() @ x}
    return {n: v.to(torch.bfloat16) for n, v in got.items()}


def run(st):
    c = st["c"]
    if own:
        from paper_2607_11185_amd import seg as S
        if c["kind"] == "pos":
            return S.seg_mrope_positions(st["problem"], st["layout"], st["grid"])
        if c["kind"] == "rope":
            f = S.seg_mrope_bwd if c["inverse"] else S.seg_mrope_fwd
            return f(st["q"], st["k"], st["pos"], S.MropeCfg((c["s0"], c["s1"], c["s2"]), 1e6))
        if c["kind"] == "act":
            return S.seg_act_unpack(S.seg_act_pack(st["x"]), st["x"].dtype)
        if not c["grad"]:
            m, kept = S.seg_glu_fwd(st["x"], st["wg"], st["wu"], keep=c["keep"])
            out = {"m": m}
            if c["keep"]:
                out["g"], out["u"] = (S.seg_act_unpack(k, torch.bfloat16) for k in kept)
            return out
        kept = tuple(S.Act8(code, exp) for code, exp in st["kept"])
        return S.seg_glu_bwd(st["x"], st["wg"], st["wu"], st["dm"], kept, dw_dtype=torch.bfloat16)
    if c["kind"] == "pos":
        return _run_pos(st)
    if c["kind"] == "rope":
        return _run_rope(st)
    if c["kind"] == "act":
        return _unpack(*_pack(st["x"].float()), st["x"].dtype)
    return _run_glu(st)


def work(c):
    if c["kind"] == "pos":
        first, rows, _, _, total = _runs(c)
        return {"bytes": 12 * total + 32 * len(rows), "flops": 0}
    if c["kind"] == "rope":
        e = 2 if c["dtype"] == "bf16" else 4
        n = c["rows"] * (c["hq"] + c["hkv"]) * c["d"]
        return {"bytes": 2 * e * n + 12 * c["rows"], "flops": 3 * n}
    if c["kind"] == "act":
        e = 2 if c["dtype"] == "bf16" else 4
        codes = c["rows"] * (c["cols"] + -(-c["cols"] // BLOCK))
        return {"bytes": 2 * e * c["rows"] * c["cols"] + 2 * codes, "flops": 4 * c["rows"] * c["cols"]}
    rows, h, i = c["rows"], c["hidden"], c["inter"]
    codes = 2 * rows * (i + -(-i // BLOCK))
    if c["grad"]:  # x, dm, weights and codes; m, dx and both weight gradients
        return {"bytes": 2 * (2 * rows * h + 2 * rows * i + 4 * i * h) + codes, "flops": 8.0 * rows * h * i}
    read_again = 2 * codes + 4 * rows * i if c["keep"] else 0
    return {"bytes": 2 * (rows * h + 2 * i * h + rows * i) + read_again, "flops": 4.0 * rows * h * i}


# ------------------------------------------------------------ exact, 64 bits

def _exact_pos(c, seed):
    """Row by row along each segment, run by run on the host."""
    first, rows, step, seg, total = _runs(c)
    grid = _grids(c, seed)
    pos = np.full((3, total), -1, np.int32)
    n, last = 0, -1
    for f, l, s, q in zip(first, rows, step, seg):
        if q != last:
            n, last = 0, q
        if s < 0:
            pos[:, f:f + l] = n + np.arange(l)
            n += l
            continue
        t, h, w, e = (int(v) for v in grid[s])
        pt, py, px = np.meshgrid(np.arange(t) * e, np.arange(h), np.arange(w), indexing="ij")
        block = np.stack([pt, py, px]).reshape(3, -1)
        pos[:, f:f + l] = n + block
        n += int(block.max()) + 1
    return torch.from_numpy(pos)


def _exact_values(v):
    """What 8 bits keep of v (64 bits): codes of at most 127 steps of the least power of two."""
    rows, cols = v.shape
    out = torch.empty_like(v)
    for at in range(0, rows, 4096):
        p = v[at:at + 4096]
        n = -(-cols // BLOCK)
        full = torch.zeros(len(p), n * BLOCK, dtype=torch.float64, device=v.device)
        full[:, :cols] = p
        full = full.view(len(p), n, BLOCK)
        top = full.abs().max(2, keepdim=True).values
        step = torch.ceil(torch.log2(top.clamp(min=2.0 ** -200) / 127)).clamp(min=-127)
        step = (step.long() + 1023 << 52).view(torch.float64)  # the power of two by its bits
        step = torch.where(top > 127 * step, step * 2, step)  # a logarithm rounded to the wrong side
        step = torch.where((top <= 63.5 * step) & (step > 2.0 ** -127), step / 2, step)
        out[at:at + 4096] = (torch.round(full / step) * step).view(len(p), -1)[:, :cols]
    return out


def exact(c, seed):
    if c["kind"] == "pos":
        return _exact_pos(c, seed)
    st = prepare(c, seed)
    if c["kind"] == "rope":
        half = c["d"] // 2
        axes = [0] * c["s0"] + [1] * c["s1"] + [2] * c["s2"]
        theta = torch.stack([st["pos"][a].double() * 1e6 ** (-2.0 * i / c["d"]) for i, a in enumerate(axes)], 1)
        turn = torch.polar(torch.ones_like(theta), -theta if c["inverse"] else theta)
        keep = (st["pos"] >= 0).all(0)
        turn[~keep] = 0 if c["inverse"] else 1
        out = []
        for x in (st["q"], st["k"]):
            y = torch.empty(x.shape, dtype=torch.float64, device=DEV)
            for head in range(x.shape[1]):
                z = torch.complex(x[:, head, :half].double(), x[:, head, half:].double()) * turn
                y[:, head, :half], y[:, head, half:] = z.real, z.imag
            out.append(y)
        return out
    if c["kind"] == "act":
        return _exact_values(st["x"].double())
    x, wg, wu = st["x"].double(), st["wg"].double(), st["wu"].double()
    if not c["grad"]:
        g, u = x @ wg.t(), x @ wu.t()
        out = {"m": g / (1 + torch.exp(-g)) * u}
        if c["keep"]:
            out["g"], out["u"] = _exact_values(g), _exact_values(u)
        return out
    g, u = (k[0].double() * (k[1].long() + 896 << 52).view(torch.float64).repeat_interleave(BLOCK, 1)[:, :c["inter"]] for k in st["kept"])
    dm = st["dm"].double()
    q = 1 / (1 + torch.exp(-g))
    silu, slope = g * q, q + g * q * (1 - q)
    dg = dm * u * slope
    du = dm * silu
    return {"m": silu * u, "dx": torch.addmm(dg @ wg, du, wu), "dwg": dg.t() @ x, "dwu": du.t() @ x}
