"""Gated feed-forward block on the GPU against the float64 oracle.

Forward: g and u are fp32 sums of exact products, off by at most e_g = (H + 1)
2^-24 sum|x w|; silu has slope at most 1.1, its fp32 evaluation is good to
(|g| + 8) 2^-23 (the exponent's argument and a few roundings); m rounds once to
bf16 (2^-8).  Kept values are off by half a step, at most max|g| / 127 of the
block, and e_g.

Backward, from given kept values: dg and du round to bf16 (2^-8), the products
are exact, their sums in fp32, the outputs round again where they are bf16.
Elementwise that is at most 2^-8 sum|dg w| + 2^-8 |out| and the sums' part; over a
whole tensor the two roundings are independent and uniform, 2^-8 / sqrt(3) each,
so the relative Frobenius error stays below 2^-8."""
import numpy as np
import pytest

from oracle import act8 as OA8
from oracle import glu as OG
from paper_2607_11185_amd import _lib
from paper_2607_11185_amd import seg as S
from tests.gpu_helpers import rel, say

pytestmark = pytest.mark.gpu

# rows, hidden, inter: one row and few, widths around the tiles of 32, 64, 128 and 256
SHAPES = [(1, 8, 8), (1, 64, 40), (3, 72, 104), (17, 328, 200), (64, 256, 256), (130, 264, 520), (300, 128, 1032),
          (257, 512, 72), (16, 1024, 2048), (33, 2048, 264),
          # each way a product is cut (test_every_way_of_cutting): parts of K and halves of tiles
          (70, 1040, 8), (674, 8, 5512), (1, 24, 320), (1624, 8, 8), (2, 8, 2712), (1813, 8, 264),
          # each kernel for few rows, K that ends inside a step and parts of K that are empty
          (2, 520, 264), (4, 1096, 96), (8, 200, 40), (5, 24, 1000), (9, 64, 256), (31, 512, 640), (50, 264, 1000), (64, 1032, 264),
          (8, 4104, 64), (1, 16384, 40)]
# whole rounds of tiles over the chip and a rest behind them
LARGE = (1500, 2048, 5504)


def _np(t):
    return t.double().cpu().numpy()


def _within(got, ref, tol, name):
    over = np.abs(got - ref) - tol
    worst = float(over.max())
    assert worst <= 0, (name, worst, int((over > 0).sum()))


def _inputs(rows, hidden, inter, seed=0, pad=0):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed * 1000 + rows)

    def r(*s, std=1.0):
        return (torch.randn(*s, generator=gen, device="cuda") * std).to(torch.bfloat16)
    x = r(rows, hidden + pad)[:, :hidden]
    return x, r(inter, hidden, std=2 / hidden ** 0.5), r(inter, hidden, std=1 / hidden ** 0.5), r(rows, inter)


def _forward_bounds(x, wg, wu):
    m, g, u = OG.forward(x, wg, wu)
    n = (x.shape[1] + 1) * 2.0 ** -24
    eg, eu = n * (np.abs(x) @ np.abs(wg).T), n * (np.abs(x) @ np.abs(wu).T)
    silu = np.abs(g * OG.sigmoid(g))
    em = 1.1 * eg * (np.abs(u) + eu) + silu * eu + silu * np.abs(u) * (np.abs(g) + 8) * 2.0 ** -23
    return m, g, u, eg, eu, em + 2.0 ** -8 * (np.abs(m) + em) + 1e-38


def _choice(rows, hidden, inter, which):
    import ctypes

    import torch  # noqa: F401  (its HIP runtime is loaded before the library asks for one)
    f = _lib.lib().seg_glu_gemm_choice
    f.restype, f.argtypes = None, [ctypes.c_int32] * 4 + [ctypes.c_void_p]
    out = (ctypes.c_int32 * 4)()
    f(rows, hidden, inter, which, out)
    tile, parts, full, rest = out
    if parts == 0:
        return f"few {tile}"
    return "whole" if not rest and parts == 1 else "parts" if not rest else ("rounds + " if full else "") + (
        "halves" if parts == 1 else "parts of the rest")


def test_every_way_of_cutting():
    """The shapes above take, for the forward, dx and the weight gradients, every way that
    their products are cut."""
    got = {(w, _choice(*s, w)) for s in [*SHAPES, LARGE] for w in range(3)}
    assert got >= {(0, f"few {n}") for n in (1, 2, 16, 32, 64)}, got
    assert got >= {(0, "whole"), (0, "parts of the rest"), (0, "rounds + parts of the rest"), (1, "whole"), (1, "parts"),
                   (1, "parts of the rest"), (2, "whole"), (2, "parts"), (2, "parts of the rest"), (2, "rounds + halves")}, got


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("shape", [*SHAPES, LARGE], ids=lambda s: "x".join(map(str, s)))
def test_forward(shape, keep):
    import torch
    rows, hidden, inter = shape
    say(shape)
    x, wg, wu, _ = _inputs(*shape, pad=8)
    m, kept = S.seg_glu_fwd(x, wg, wu, keep=keep)
    ref, g, u, eg, eu, em = _forward_bounds(_np(x), _np(wg), _np(wu))
    _within(_np(m), ref, em, "m")
    assert (kept is not None) == keep
    for a, v, e in zip(kept or (), (g, u), (eg, eu)):
        got = _np(S.seg_act_unpack(a, torch.float32))
        top = np.abs(np.pad(v, ((0, 0), (0, -inter % 32)))).reshape(rows, -1, 32).max(-1)
        top = np.repeat(top, 32, 1)[:, :inter]
        _within(got, v, (top + e) / 127 + e, "kept")
    if keep:
        assert torch.equal(m, S.seg_glu_fwd(x, wg, wu)[0])     # the same m either way


def _kept_of(g, u):
    import torch
    out = []
    for v in (g, u):
        code, exp = OA8.pack(v)
        out.append(S.Act8(torch.from_numpy(code).cuda(), torch.from_numpy(exp).cuda()))
    return tuple(out), tuple(OA8.unpack(*OA8.pack(v)) for v in (g, u))


@pytest.mark.parametrize("dw", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [*SHAPES, LARGE], ids=lambda s: "x".join(map(str, s)))
def test_backward_from_kept_values(shape, dw):
    import torch
    rows, hidden, inter = shape
    x, wg, wu, dm = _inputs(*shape, seed=1, pad=16)
    xn, wgn, wun, dmn = (_np(t) for t in (x, wg, wu, dm))
    _, g, u = OG.forward(xn, wgn, wun)
    kept, (gv, uv) = _kept_of(g, u)
    out = S.seg_glu_bwd(x, wg, wu, dm, kept, dw_dtype=torch.bfloat16 if dw == "bf16" else torch.float32)
    dg, du = OG.backward_act(gv, uv, dmn)
    dx, dwg, dwu = OG.backward(xn, wgn, wun, gv, uv, dmn)
    h = 2.0 ** -8
    ag, au = np.abs(dg), np.abs(du)
    # the activation's own fp32 error joins the rounding of dg and du
    ag_e, au_e = ag * h + (np.abs(dmn * uv) * (np.abs(gv) + 8) * 2.0 ** -22), au * h + (np.abs(dmn * gv) * 2.0 ** -22)
    n = (2 * inter + 1) * 2.0 ** -24
    sums = (ag + ag_e) @ np.abs(wgn) + (au + au_e) @ np.abs(wun)
    checks = [("dx", dx, ag_e @ np.abs(wgn) + au_e @ np.abs(wun) + n * sums, True)]
    n = (rows + 1) * 2.0 ** -24
    for name, ref, e, a in (("dwg", dwg, ag_e, ag), ("dwu", dwu, au_e, au)):
        checks.append((name, ref, e.T @ np.abs(xn) + n * ((a + e).T @ np.abs(xn)), dw == "bf16"))
    for name, ref, tol, bf in checks:
        got = _np(out[name])
        tol = tol + (h * (np.abs(ref) + tol) if bf else 0) + 1e-38
        _within(got, ref, tol, name)
        if ref.size >= 4096:
            assert rel(got, ref) < h, (name, rel(got, ref))
    m = gv * OG.sigmoid(gv) * uv
    _within(_np(out["m"]), m, h * np.abs(m) * (1 + 1e-5) + np.abs(m) * (np.abs(gv) + 8) * 2.0 ** -22 + 1e-38, "m")


# (a kernel for few rows, for some tens, the GEMM whole and in parts: each in its bf16 form)
@pytest.mark.parametrize("shape", [(17, 328, 200), (300, 128, 1032), (3, 520, 136), (70, 1040, 40), (7, 256, 264)], ids=str)
def test_backward_without_kept_values(shape):
    """Gate and up values computed again, in bf16: their rounding (2^-8) moves dg and du
    by a few times that, independently, so 2^-6 bounds the relative Frobenius error."""
    import torch
    x, wg, wu, dm = _inputs(*shape, seed=2)
    xn, wgn, wun, dmn = (_np(t) for t in (x, wg, wu, dm))
    m, g, u = OG.forward(xn, wgn, wun)
    out = S.seg_glu_bwd(x, wg, wu, dm, None)
    for name, ref in zip(("dx", "dwg", "dwu", "m"), (*OG.backward(xn, wgn, wun, g, u, dmn), m)):
        assert rel(_np(out[name]), ref) < 2.0 ** -6, name
    only = S.seg_glu_bwd(x, wg, wu, dm, None, want_m=False)
    assert only["m"] is None and all(torch.equal(only[n], out[n]) for n in ("dx", "dwg", "dwu"))


def test_forward_and_backward_as_used():
    """The kept values of a forward through the backward: gradients of the block within
    what 8 bits take (steps of at most 2 / 127 of a block's largest value, about 1 % of a
    value in the mean, twice where g enters as product and slope)."""
    shape = (200, 256, 512)
    x, wg, wu, dm = _inputs(*shape, seed=3)
    m, kept = S.seg_glu_fwd(x, wg, wu, keep=True)
    out = S.seg_glu_bwd(x, wg, wu, dm, kept)
    xn, wgn, wun, dmn = (_np(t) for t in (x, wg, wu, dm))
    _, g, u = OG.forward(xn, wgn, wun)
    for name, ref in zip(("dx", "dwg", "dwu"), OG.backward(xn, wgn, wun, g, u, dmn)):
        assert rel(_np(out[name]), ref) < 2.0 / 63.5, name
    assert rel(_np(out["m"]), _np(m)) < 2.0 / 63.5


def test_extremes():
    """A row of zeros, gates far from zero on both sides, and an infinity that stays in its row."""
    import torch
    x, wg, wu, dm = _inputs(40, 64, 96, seed=4)
    x[3] = 0
    x[4] *= 100
    m, kept = S.seg_glu_fwd(x, wg, wu, keep=True)
    assert not m[3].any() and not kept[0].exp[3].any() and not kept[1].code[3].any()
    ref = OG.forward(*(_np(t) for t in (x, wg, wu)))[0]
    assert rel(_np(m)[4], ref[4]) < 2.0 ** -8
    x[7, 5] = float("inf")
    m2, kept2 = S.seg_glu_fwd(x, wg, wu, keep=True)
    rows = torch.arange(40, device="cuda") != 7
    assert torch.equal(m2[rows], m[rows]) and bool((kept2[0].exp[7] == 255).all())
    assert torch.equal(kept2[0].code[rows], kept[0].code[rows])


@pytest.mark.parametrize("shape", [(2, 328, 104), (5, 328, 104), (16, 1096, 40), (30, 1096, 104), (50, 328, 72), (300, 328, 104)],
                         ids=str)
def test_infinities_stay_in_their_row_and_feature(shape):
    """An infinite row of x and a NaN in a weight reach that row's and that feature's values
    only, though rows and features share loads, LDS and matrix operands."""
    import torch
    rows, hidden, inter = shape
    x, wg, wu, _ = _inputs(*shape, seed=6)
    m = S.seg_glu_fwd(x, wg, wu)[0]
    x2, w2 = x.clone(), wu.clone()
    x2[rows - 1, hidden - 3] = float("inf")
    w2[inter - 2, 7] = float("nan")
    m2 = S.seg_glu_fwd(x2, wg, w2)[0]
    assert torch.equal(m2[:-1, :-2], m[:-1, :-2]) and torch.equal(m2[:-1, -1], m[:-1, -1])
    assert bool(m2[:, -2].isnan().all()) and not bool(m2[-1].isfinite().all())


@pytest.mark.parametrize("rows", [1, 22, 300])
def test_gates_over_the_whole_range(rows):
    """g = x[:, 0] and u = 1 exactly, down to where exp(-g) leaves fp32: there the sigmoid
    may be off by 2^-126, elsewhere by the exponential's and four more roundings."""
    import torch
    steps = [0, 2.0 ** -120, 1e-3, 1, 1.28125, 5, 20, 80, 87, 87.5, 88, 88.5, 89, 104, 1e4, 3e38]
    v = torch.tensor([s * t for t in steps for s in (1, -1)]).to(torch.bfloat16)
    for v in v.split(1) if rows == 1 else [v.repeat(-(-rows // len(v)))[-rows:]]:
        x = torch.zeros(len(v), 64, dtype=torch.bfloat16)
        x[:, 0], x[:, 1] = v, 1
        wg, wu = torch.zeros(2, 64, 64, dtype=torch.bfloat16)
        wg[:, 0] = wu[:, 1] = 1
        x, wg, wu = x.cuda(), wg.cuda(), wu.cuda()
        m, kept = S.seg_glu_fwd(x, wg, wu, keep=True)
        g = v.double().numpy()
        for g, name in ((g, "m"), (_np(S.seg_act_unpack(kept[0], torch.float32))[:, 0], "dx")):
            with np.errstate(over="ignore"):
                s, c = OG.sigmoid(g), np.minimum(np.abs(g), 110)  # past 110 the sigmoid is 0 or 1
            es = s * ((1 - s) * (c + 8) + 2) * 2.0 ** -23 + (g < -87.3) * 2.0 ** -126
            em = c * es + 2.0 ** -8 * np.abs(g * s) + 2.0 ** -133
            if name == "m":
                _within(_np(m), (g * s)[:, None], em[:, None] * 1.01, name)
                continue
            # from the kept g (8 bits: not x's own); 64 equal terms, their sum rounded again
            dx = _np(S.seg_glu_bwd(x, wg, wu, torch.ones_like(m), kept)["dx"])
            d = s * (1 + g * (1 - s))
            ed = es * (1 + 2 * c) + s * (1 + c * (1 - s)) * 2.0 ** -22 + 2.0 ** -8 * np.abs(d) + 2.0 ** -133
            for at, ref, e in ((0, d, ed), (1, g * s, em)):
                fits = np.abs(ref) < 4e36
                got = np.where(fits, dx[:, at], 64 * ref)
                _within(got, 64 * ref, 64 * 1.01 * (e + 2.0 ** -8 * np.abs(ref)), at)


def test_no_rows_give_zero_weight_gradients():
    import torch
    x, wg, wu, dm = _inputs(4, 64, 72)
    assert S.seg_glu_fwd(x[:0], wg, wu, keep=True)[0].shape == (0, 72)
    for dt in (torch.bfloat16, torch.float32):
        nan = {n: torch.full((72, 64), float("nan"), dtype=dt, device="cuda") for n in ("dwg", "dwu")}
        S.seg_glu_bwd(x[:0], wg, wu, dm[:0], None, out=dict(nan, dx=x[:0].contiguous(), m=None))
        assert not nan["dwg"].any() and not nan["dwu"].any()


@pytest.mark.parametrize("shape", [(1, 64, 40), (3, 72, 104), (17, 328, 200), (130, 264, 520), (257, 512, 72), (70, 1040, 8),
                                   LARGE], ids=str)
def test_nothing_is_written_past_the_end(shape):
    """Outputs as the first part of larger buffers, workspaces of exactly the size that is asked
    for: what lies behind stays as it was."""
    import torch
    rows, hidden, inter = shape
    x, wg, wu, dm = _inputs(*shape, seed=6)

    def room(shape, dtype):
        n = int(np.prod(shape))
        flat = torch.full((n + 4096,), 77, dtype=dtype, device="cuda")
        return flat[:n].view(shape), flat[n:]
    bf, nb = torch.bfloat16, -(-inter // 32)
    m, m_end = room((rows, inter), bf)
    codes = [room((rows, inter), torch.int8) for _ in range(2)]
    exps = [room((rows, nb), torch.uint8) for _ in range(2)]
    kept = tuple(S.Act8(c[0], e[0]) for c, e in zip(codes, exps))
    ends = [m_end, *(c[1] for c in codes), *(e[1] for e in exps)]
    ws, end = room((S.glu_workspace(*shape, False, False, "cuda").numel(),), torch.uint8)
    S.seg_glu_fwd(x, wg, wu, keep=kept, m=m, ws=ws)
    ends.append(end)
    for k in (kept, None):
        for dt in (bf, torch.float32):
            out = {n: room(s, t) for n, s, t in (("dx", (rows, hidden), bf), ("dwg", (inter, hidden), dt),
                                                 ("dwu", (inter, hidden), dt), ("m", (rows, inter), bf))}
            ws, end = room((S.glu_workspace(*shape, True, k is not None, "cuda").numel(),), torch.uint8)
            S.seg_glu_bwd(x, wg, wu, dm, k, out={n: t[0] for n, t in out.items()}, ws=ws)
            ends += [end, *(t[1] for t in out.values())]
    for i, e in enumerate(ends):
        assert bool((e == 77).all()), i


@pytest.mark.parametrize("rows,hidden,inter", [(1, 64, 40), (22, 64, 64), (300, 64, 64), (70, 1040, 8)],
                         ids=["few", "rows", "product", "product in parts"])
def test_sigmoid_where_it_is_subnormal(rows, hidden, inter):
    """Gates of -87.4 to -88.5: the sigmoid is a subnormal number there (a step of 2^-149), and
    times g an ordinary one.  g = -(88 + t) exactly, u = 1; the exponential is off by the
    rounding of its argument and a few more (|g| + 8) 2^-23."""
    import torch
    t = (torch.arange(rows) * 37 % 72 - 38) / 64.0       # -38/64 .. 33/64
    if rows == 1:
        t[0] = 0.25
    x = torch.zeros(rows, hidden)
    x[:, 0], x[:, 1], x[:, 2] = -88, 1, -t
    wg, wu = torch.zeros(2, inter, hidden)
    wg[:, 0] = wg[:, 2] = wu[:, 1] = 1
    x, wg, wu = (v.to(torch.bfloat16).cuda() for v in (x, wg, wu))
    m, kept = S.seg_glu_fwd(x, wg, wu, keep=True)
    g = -88 - t.double().numpy()
    ref = g * OG.sigmoid(g)
    tol = np.abs(ref) * ((np.abs(g) + 8) * 2.0 ** -23 + 2.0 ** -8) * 1.01 + np.abs(g) * 2.0 ** -149 + 2.0 ** -133
    assert np.abs(ref).min() > 2 * tol.max()             # zeros would not pass
    _within(_np(m), ref[:, None], tol[:, None], "m")
    # backward: the kept g has steps of one, half a step off -88.52 .. -87.40: -87, -88 or -89
    assert bool((S.seg_act_unpack(kept[0], torch.float32)[:, 0] + 88).abs().max() <= 1)
    out = S.seg_glu_bwd(x, wg, wu, torch.ones_like(m), kept)
    g = _np(S.seg_act_unpack(kept[0], torch.float32))[:, 0]
    ok = g == -88
    ref = (g * OG.sigmoid(g))[ok]
    tol = np.abs(ref) * ((np.abs(g[ok]) + 8) * 2.0 ** -23 + 2.0 ** -8) * 1.01 + np.abs(g[ok]) * 2.0 ** -149 + 2.0 ** -133
    assert ok.any()
    _within(_np(out["m"])[ok], ref[:, None], tol[:, None], "m of the backward")


# Launches that the shapes above leave out, each with ragged last tiles: rows, hidden, inter
REST = [(136, 344, 33896), (10847, 6848, 8), (41876, 5120, 136), (8274, 8, 1256), (35082, 272, 136), (5057, 3104, 360),
        (5648, 3472, 2408), (32792, 8, 8), (1809, 8, 5392), (727, 8, 33432), (7304, 264, 19128), (66, 8, 16576)]


def _launch(rows, hidden, inter, which):
    """The way a product is cut and the rows of its (rest's) tiles."""
    import ctypes
    way = _choice(rows, hidden, inter, which)
    out = (ctypes.c_int32 * 4)()
    _lib.lib().seg_glu_gemm_choice(rows, hidden, inter, which, out)
    return which, way, out[0]


def test_every_launch_is_tested():
    """With both tile heights: the forward, dx and the weight gradients uncut, in parts of K, and
    as whole rounds of tiles with a rest in halves of tiles or in parts of K."""
    got = {_launch(*s, w) for s in [*SHAPES, LARGE, *REST] for w in range(3)}
    few = {(0, f"few {n}", n) for n in (1, 2, 16, 32, 64)}
    ways = {(w, way, t) for w in range(3) for t in (128, 256) for way in ("whole", "parts", "rounds + parts of the rest")}
    ways |= {(w, "rounds + halves", 128) for w in range(3)} | {(w, "parts of the rest", 128) for w in range(3)}
    ways |= {(0, "parts of the rest", 256)}
    ways -= {(0, "parts", 128), (0, "parts", 256)}      # of the forward all tiles are a rest then
    assert got >= few | ways, (few | ways) - got
    # sizes of the timing cases and of the decoder layer's classes bring no others
    more = {_launch(r, h, i, w) for r in (1, 4, 65, 100, 300, 1000, 1500, 3000, 4096, 8192, 16384, 65536, 138819)
            for h, i in ((896, 4864), (1536, 8960), (2048, 5504), (3584, 18944), (4096, 14336), (8192, 28672)) for w in range(3)}
    assert more <= got, more - got


def _over(got, ref, tol, name):
    worst = float((got.double() - ref).abs().sub_(tol).max())
    assert worst <= 0, (name, worst)


@pytest.mark.parametrize("shape", REST, ids=lambda s: "x".join(map(str, s)))
def test_launches_of_larger_products(shape):
    """Forward, with and without kept values, and backward from kept values with both types of
    weight gradients, against products in 64 bits on the GPU; bounds as above."""
    import torch
    rows, hidden, inter = shape
    say(shape, [_launch(*shape, w)[1:] for w in range(3)])
    x, wg, wu, dm = _inputs(*shape, seed=7, pad=8)
    xd, wgd, wud, dmd = (t.double() for t in (x, wg, wu, dm))
    h = 2.0 ** -8
    g, u = xd @ wgd.t(), xd @ wud.t()
    n = (hidden + 1) * 2.0 ** -24
    eg, eu = n * (xd.abs() @ wgd.abs().t()), n * (xd.abs() @ wud.abs().t())
    silu = g * torch.sigmoid(g)
    em = 1.1 * eg * (u.abs() + eu) + silu.abs() * eu + (silu * u).abs() * (g.abs() + 8) * 2.0 ** -23
    m, kept = S.seg_glu_fwd(x, wg, wu, keep=True)
    _over(m, silu * u, em + h * ((silu * u).abs() + em) + 1e-38, "m")
    assert torch.equal(m, S.seg_glu_fwd(x, wg, wu)[0])
    del silu, em
    for a, v, e in zip(kept, (g, u), (eg, eu)):
        top = torch.nn.functional.pad(v.abs(), (0, -inter % 32)).view(rows, -1, 32).amax(-1).repeat_interleave(32, 1)[:, :inter]
        _over(S.seg_act_unpack(a, torch.float32), v, (top + e) / 127 + e, "kept")
    del g, u, eg, eu, top
    gv, uv = (S.seg_act_unpack(a, torch.float32).double() for a in kept)
    s = torch.sigmoid(gv)
    dg, du = dmd * uv * s * (1 + gv * (1 - s)), dmd * gv * s
    ge = dg.abs() * h + (dmd * uv).abs() * (gv.abs() + 8) * 2.0 ** -22
    ue = du.abs() * h + (dmd * gv).abs() * 2.0 ** -22
    ga, ua = dg.abs() + ge, du.abs() + ue
    want = {"dx": (dg @ wgd + du @ wud,
                   ge @ wgd.abs() + ue @ wud.abs() + (2 * inter + 1) * 2.0 ** -24 * (ga @ wgd.abs() + ua @ wud.abs()))}
    for name, d, e, a in (("dwg", dg, ge, ga), ("dwu", du, ue, ua)):
        want[name] = d.t() @ xd, (e + (rows + 1) * 2.0 ** -24 * a).t() @ xd.abs()
    del dg, du, ge, ue, ga, ua, s, gv, uv
    for dt in (torch.bfloat16, torch.float32):
        out = S.seg_glu_bwd(x, wg, wu, dm, kept, dw_dtype=dt)
        for name, (ref, tol) in want.items():
            more = h * (ref.abs() + tol) if out[name].dtype == torch.bfloat16 else 0
            _over(out[name], ref, tol + more + 1e-38, name)


@pytest.mark.parametrize("shape", [(1, 328, 104), (2, 328, 104), (5, 328, 104), (16, 1096, 40), (30, 1096, 104), (50, 328, 72),
                                   (300, 328, 104), (70, 1040, 40)], ids=str)
def test_an_infinity_reaches_its_whole_row(shape):
    """An infinity of x makes every feature of its row non-finite: g and u are infinities or (a
    weight of zero) NaN, and silu of an infinity times one is an infinity or NaN."""
    import torch
    rows, hidden, inter = shape
    x, wg, wu, _ = _inputs(*shape, seed=6)
    for k in (0, hidden - 3, hidden - 1):
        x2 = x.clone()
        x2[rows - 1, k] = float("inf")
        m = S.seg_glu_fwd(x2, wg, wu)[0]
        assert bool(m[:-1].isfinite().all()) and not bool(m[-1].isfinite().any()), k
