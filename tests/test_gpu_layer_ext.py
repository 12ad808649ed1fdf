"""The decoder layer with positions on three axes and 8-bit saved activations
(seg_layer_fwd_ext / seg_layer_bwd_ext): against the float64 oracle layer, and
against the parts it is made of, bit for bit."""
import numpy as np
import pytest

from oracle import act8 as OA8
from oracle import layer as OLY
from oracle import layout as OL
from oracle import mrope as OM
from paper_2607_11185_amd import _lib
from paper_2607_11185_amd import seg as S
from paper_2607_11185_amd import workload as WL
from tests.gpu_helpers import TOL, rel, say, vis_window
from tests.test_gpu_layer import BASE, EPS, MED, LayerRun, _np

pytestmark = pytest.mark.gpu

# screenshots of 150 tokens are 10 x 15 patches, or clips of 2 frames of 5 x 15
CASES = {
    "d64_gqa2_ragged": (MED, 328, 200, 0, (8, 12, 12)),
    "d128_chunked": (MED.with_(head_dim=128, seed=1), 256, 688, 300, (16, 24, 24)),
    "d64_gqa4_buffers": (MED.with_(hq=8, hkv=2, buffer_tokens=1400, seed=2, steps=(3, 5)), 384, 520, 512, (32, 0, 0)),
    "anchored_k2_d3": (MED.with_(mode="anchored", window=2, seg_steps=3, seed=4, steps=(8, 9)), 264, 320, 0, (0, 5, 27)),
}


class ExtRun(LayerRun):
    def __init__(self, cfg, H, I, chunk, sections):
        import torch
        super().__init__(cfg, H, I, chunk)
        rng = np.random.default_rng(cfg.seed)
        n = self.run.spans.num_steps
        self.grid = np.where((rng.random(n) < 0.5)[:, None], [[1, 10, 15, 1]], [[2, 5, 15, 3]]).astype(np.int32)
        self.rope = S.MropeCfg(sections, BASE)
        self.pos = S.seg_mrope_positions(self.run.problem, self.lay, self.grid)
        # what lies in padding rows does not count
        pad = torch.from_numpy(self.run.host["tok_src"] < 0).to(self.dev)
        self.pad = pad
        self.x[pad] = float("nan")
        self.dy[pad] = float("inf")
        self.pos[:, pad] = 77

    def oracle_parts(self):
        c = self.cfg
        ref = OL.build(self.run.spans, c.window, c.seg_steps, 128, c.max_seg_tokens, c.buffer_tokens, with_tiles=False,
                       mode=c.mode)
        pos = np.maximum(OM.positions(ref, self.run.spans, self.grid, ref.packed_tokens), 0)
        x = WL.layer_rows_np(self.seed, "x", self.src, self.H)
        x[ref.tok_src < 0] = 0
        dy = WL.layer_rows_np(self.seed, "dy", np.arange(self.P), self.H)
        w = OLY.Weights(**WL.layer_weights_np(self.seed, self.H, self.I, c.hq, c.hkv, c.head_dim))
        masks = [OL.visibility(sg, vis_window(c)) for sg in ref.segments]
        a = dict(hq=c.hq, hkv=c.hkv, d=c.head_dim, eps=EPS, base=BASE,
                 rot=lambda t, inverse: OM.rotate(t, pos, self.rope.sections, BASE, inverse))
        return x, w, ref, masks, a, dy


def _rows(pad, t):
    return t[~pad]


@pytest.mark.parametrize("name", list(CASES))
def test_three_axes_full_parity(name):
    """y, dx and all weight gradients against the oracle with three-axis rotation."""
    say(name)
    lr = ExtRun(*CASES[name])
    y, saved = S.seg_layer_fwd_ext(lr.lay, lr.lc, lr.w, lr.x, lr.rope, lr.pos)
    dx, grads = S.seg_layer_bwd_ext(lr.lay, lr.lc, lr.w, lr.dy, lr.rope, lr.pos, x=lr.x, saved=saved)
    x, w, ref, masks, a, dy = lr.oracle_parts()
    y_ref, sv = OLY.forward(x, w, ref.segments, masks, **a)
    dx_ref, g_ref = OLY.backward(x, w, ref.segments, masks, **a, saved=sv, dy=dy)
    ok = ref.tok_src >= 0
    assert rel(_np(y)[ok], y_ref[ok]) < TOL and rel(_np(saved["q"])[ok], sv["qr"][ok]) < TOL
    assert rel(_np(dx)[ok], dx_ref[ok]) < TOL and not dx[lr.pad].any()
    for n in _lib.LAYER_WEIGHTS:
        assert rel(_np(grads[n]), g_ref[n]) < TOL, n


@pytest.mark.parametrize("keep_gate", [False, True])
@pytest.mark.parametrize("name", list(CASES))
def test_saved_in_8_bits(name, keep_gate):
    """The forward's output is that without; what is kept is the packed form of what the
    layer saves in bf16; the backward is the layer's on the kept values: bit for bit
    where the gate and up values are computed again, against the oracle on the same kept
    values where they are kept."""
    import torch
    say(name, keep_gate)
    lr = ExtRun(*CASES[name])
    H = lr.H
    y, saved = S.seg_layer_fwd_ext(lr.lay, lr.lc, lr.w, lr.x, lr.rope, lr.pos)
    s8 = S.layer_saved8(lr.lay, lr.lc, keep_gate)
    y8, back = S.seg_layer_fwd_ext(lr.lay, lr.lc, lr.w, lr.x, lr.rope, lr.pos, saved8=s8)
    assert back is s8 and torch.equal(_rows(lr.pad, y8), _rows(lr.pad, y))
    for n in ("lse", "rstd1", "rstd2"):
        t, u = (s8[n], saved[n]) if n != "lse" else (s8[n].T, saved[n].T)
        assert torch.equal(_rows(lr.pad, t), _rows(lr.pad, u)), n
    for n in ("x", "q", "k", "v", "o", "y1"):
        t = lr.x if n == "x" else saved[n].reshape(lr.P, -1)
        want = S.seg_act_pack(t)
        assert torch.equal(_rows(lr.pad, s8[n].code), _rows(lr.pad, want.code)), n
        assert torch.equal(_rows(lr.pad, s8[n].exp), _rows(lr.pad, want.exp)), n
    dx, grads = S.seg_layer_bwd_ext(lr.lay, lr.lc, lr.w, lr.dy, lr.rope, lr.pos, saved8=s8)
    c = lr.cfg
    val = {n: S.seg_act_unpack(s8[n]) for n in ("x", "q", "k", "v", "o", "y1")}
    if not keep_gate:
        sv = {"q": val["q"].view(lr.P, c.hq, -1), "k": val["k"].view(lr.P, c.hkv, -1), "v": val["v"].view(lr.P, c.hkv, -1),
              "o": val["o"].view(lr.P, c.hq, -1), "y1": val["y1"], **{n: s8[n] for n in ("lse", "rstd1", "rstd2")}}
        dx1, g1 = S.seg_layer_bwd_ext(lr.lay, lr.lc, lr.w, lr.dy, lr.rope, lr.pos, x=val["x"], saved=sv)
        assert torch.equal(dx, dx1)
        for n in _lib.LAYER_WEIGHTS:
            assert torch.equal(grads[n], g1[n]), n
        return
    x, w, ref, masks, a, dy = lr.oracle_parts()
    ok = ref.tok_src >= 0

    def f(t, *shape):
        t = _np(t)
        t[~ok] = 0
        return t.reshape(lr.P, *shape) if shape else t
    pos = OLY.segment_positions(ref.segments, lr.P)
    r1, r2 = (np.where(ok, _np(s8[n]), 0) for n in ("rstd1", "rstd2"))
    sv = dict(pos=pos, a=f(val["x"]) * r1[:, None] * w.g1, r1=r1, qr=f(val["q"], c.hq, c.head_dim), kr=f(val["k"], c.hkv, c.head_dim),
              v=f(val["v"], c.hkv, c.head_dim), o=f(val["o"], c.hq, c.head_dim), y1=f(val["y1"]),
              b=f(val["y1"]) * r2[:, None] * w.g2, r2=r2, gt=f(S.seg_act_unpack(s8["g"])), ut=f(S.seg_act_unpack(s8["u"])))
    sv["mm"] = OLY.silu(sv["gt"]) * sv["ut"]
    dx_ref, g_ref = OLY.backward(f(val["x"]), w, ref.segments, masks, **a, saved=sv, dy=dy)
    # the layer forms rstd from the kept x and y1 again, and the scores from the kept q and k
    # against the forward's lse: both are off by at most the 8 bits' 1 % of a value
    assert rel(_np(dx)[ok], dx_ref[ok]) < 2 * TOL and not dx[lr.pad].any()
    for n in _lib.LAYER_WEIGHTS:
        assert rel(_np(grads[n]), g_ref[n]) < 2 * TOL, n


def test_gradients_next_to_those_in_bf16():
    """What 8 bits cost: gradients against the layer's own in bf16.  Each kept value is off by
    at most 1 / 127 of its block's largest, about 1 % of a value of normal blocks, and six
    of them enter a gradient: below 6 %."""
    lr = ExtRun(*CASES["d128_chunked"])
    y, saved = S.seg_layer_fwd_ext(lr.lay, lr.lc, lr.w, lr.x, lr.rope, lr.pos)
    dx, grads = S.seg_layer_bwd_ext(lr.lay, lr.lc, lr.w, lr.dy, lr.rope, lr.pos, x=lr.x, saved=saved)
    for keep in (False, True):
        s8 = S.layer_saved8(lr.lay, lr.lc, keep)
        S.seg_layer_fwd_ext(lr.lay, lr.lc, lr.w, lr.x, lr.rope, lr.pos, saved8=s8)
        dx8, g8 = S.seg_layer_bwd_ext(lr.lay, lr.lc, lr.w, lr.dy, lr.rope, lr.pos, saved8=s8)
        assert rel(_np(dx8), _np(dx)) < 0.06
        for n in _lib.LAYER_WEIGHTS:
            say(keep, n, rel(_np(g8[n]), _np(grads[n])))
            assert rel(_np(g8[n]), _np(grads[n])) < 0.06, n


def test_without_extensions_it_is_the_layer():
    import torch
    lr = LayerRun(*CASES["d64_gqa4_buffers"][:4])
    y, saved, dx, grads = lr.gpu()
    y2, saved2 = S.seg_layer_fwd_ext(lr.lay, lr.lc, lr.w, lr.x)
    dx2, grads2 = S.seg_layer_bwd_ext(lr.lay, lr.lc, lr.w, lr.dy, x=lr.x, saved=saved2)
    pad = torch.from_numpy(lr.run.host["tok_src"] < 0).to(lr.dev)
    assert torch.equal(_rows(pad, y), _rows(pad, y2)) and torch.equal(dx, dx2)
    assert all(torch.equal(grads[n], grads2[n]) for n in grads)


def test_three_axes_all_equal_are_the_row():
    """Positions equal to the row in the segment on every axis: the layer's own embedding, up
    to the last bits of its angles (fp32 sines of two roundings)."""
    lr = ExtRun(*CASES["d128_chunked"])
    row = OLY.segment_positions(OL.build(lr.run.spans, lr.cfg.window, lr.cfg.seg_steps, 128, with_tiles=False).segments, lr.P)
    import torch
    pos = torch.from_numpy(np.stack([row] * 3).astype(np.int32)).to(lr.dev)
    y, saved = S.seg_layer_fwd_ext(lr.lay, lr.lc, lr.w, lr.x, S.MropeCfg((16, 24, 24), BASE), pos)
    y2, saved2 = S.seg_layer_fwd(lr.lay, lr.lc, lr.w, lr.x)
    assert rel(_np(saved["q"]), _np(saved2["q"])) < 2.0 ** -9 and rel(_np(y), _np(y2)) < 2.0 ** -8


def test_chunking_leaves_what_is_kept_unchanged():
    import torch
    cfg, H, I, _, sections = CASES["d64_gqa4_buffers"]
    kept = []
    for chunk in (0, 97):
        lr = ExtRun(cfg, H, I, chunk, sections)
        s8 = S.layer_saved8(lr.lay, lr.lc, True)
        y, _ = S.seg_layer_fwd_ext(lr.lay, lr.lc, lr.w, lr.x, lr.rope, lr.pos, saved8=s8)
        kept.append((y, s8))
    pad = lr.pad
    assert torch.equal(_rows(pad, kept[0][0]), _rows(pad, kept[1][0]))
    for n in _lib.SAVED8:
        for f in ("code", "exp"):
            assert torch.equal(_rows(pad, getattr(kept[0][1][n], f)), _rows(pad, getattr(kept[1][1][n], f))), (n, f)


@pytest.mark.parametrize("keep_gate", [False, True])
def test_workspaces_of_the_size_asked_for(keep_gate):
    """Nothing is read or written behind a workspace of exactly that size."""
    import torch
    lr = ExtRun(*CASES["d64_gqa4_buffers"])
    res = []
    for fill in (0, 255):
        s8 = S.layer_saved8(lr.lay, lr.lc, keep_gate)
        sizes = [S.layer_ext_workspace(lr.lay, lr.lc, True, b).numel() for b in (False, True)]
        ws = [torch.full((n + 65536,), fill, dtype=torch.uint8, device=lr.dev) for n in sizes]
        y, _ = S.seg_layer_fwd_ext(lr.lay, lr.lc, lr.w, lr.x, lr.rope, lr.pos, saved8=s8, ws=ws[0][:sizes[0]])
        dx, g = S.seg_layer_bwd_ext(lr.lay, lr.lc, lr.w, lr.dy, lr.rope, lr.pos, saved8=s8, ws=ws[1][:sizes[1]])
        assert all(bool((w[n:] == fill).all()) for w, n in zip(ws, sizes))
        res.append([_rows(lr.pad, y), dx, *g.values()])
    assert all(torch.equal(a, b) for a, b in zip(*res))


def test_capture_and_replay_of_the_operators_together():
    """Rotation, packing, the gated block and the extended layer in one graph, replayed
    between eager work: every replay equals the eager run."""
    import torch
    lr = ExtRun(*CASES["d64_gqa4_buffers"])
    H, I = lr.H, lr.I
    x2 = torch.randn(150, H, device=lr.dev, generator=torch.Generator(device=lr.dev).manual_seed(3)).to(torch.bfloat16)
    dm = torch.randn(150, I, device=lr.dev, generator=torch.Generator(device=lr.dev).manual_seed(4)).to(torch.bfloat16)
    qk = torch.randn(150, 6, 64, device=lr.dev, generator=torch.Generator(device=lr.dev).manual_seed(5))
    pos = lr.pos[:, :150].contiguous()

    def step():
        s8 = S.layer_saved8(lr.lay, lr.lc, True)
        y, _ = S.seg_layer_fwd_ext(lr.lay, lr.lc, lr.w, lr.x, lr.rope, lr.pos, saved8=s8)
        dx, grads = S.seg_layer_bwd_ext(lr.lay, lr.lc, lr.w, lr.dy, lr.rope, lr.pos, saved8=s8)
        q, k = S.seg_mrope_fwd(qk[:, :4], qk[:, 4:], pos, lr.rope)
        xv = S.seg_act_unpack(S.seg_act_pack(x2))
        m, kept = S.seg_glu_fwd(xv, lr.w["wg"], lr.w["wu"], keep=True)
        g = S.seg_glu_bwd(xv, lr.w["wg"], lr.w["wu"], dm, kept)
        return {"y": y, "dx": dx, "q": q, "k": k, "xv": xv, "m": m, **{"l" + n: t for n, t in grads.items()},
                **{"b" + n: t for n, t in g.items()}}
    eager = {n: t.clone() for n, t in step().items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    scratch = torch.randn(1 << 20, device=lr.dev)
    for rep in range(3):
        scratch.mul_(1.0001).add_(0.5)
        torch.cuda.synchronize()
        for t in out.values():
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for n, t in out.items():
            if n == "y":
                t, e = _rows(lr.pad, t), _rows(lr.pad, eager[n])
            else:
                e = eager[n]
            assert torch.equal(t, e), (rep, n)
        say("replay", rep)


@pytest.mark.parametrize("keep_gate", [False, True])
@pytest.mark.parametrize("name", ["d128_chunked", "d64_gqa4_buffers"])
def test_output_in_place_of_the_input(name, keep_gate):
    """With 8-bit saved activations y may be x and dx may be dy: what is kept, both outputs and
    all gradients are those of separate tensors, bit for bit."""
    import torch
    say(name, keep_gate)
    lr = ExtRun(*CASES[name])
    res = []
    for inplace in (False, True):
        x, dy, s8 = lr.x.clone(), lr.dy.clone(), S.layer_saved8(lr.lay, lr.lc, keep_gate)
        y, _ = S.seg_layer_fwd_ext(lr.lay, lr.lc, lr.w, x, lr.rope, lr.pos, saved8=s8, y=x if inplace else None)
        dx, g = S.seg_layer_bwd_ext(lr.lay, lr.lc, lr.w, dy, lr.rope, lr.pos, saved8=s8, dx=dy if inplace else None)
        assert (y is x) == inplace and (dx is dy) == inplace
        kept = {n + " " + f: _rows(lr.pad, getattr(s8[n], f)) for n in _lib.SAVED8 if n in s8 for f in ("code", "exp")}
        res.append({"y": _rows(lr.pad, y), "dx": dx, **kept, **{"d" + n: t for n, t in g.items()}})
    for n in res[0]:
        assert torch.equal(res[0][n], res[1][n]), n


def test_timing_counts_each_kernel_once():
    """The layer's packing and unpacking are under "ly_act8", the operators' own calls under their
    names, and calls that are refused or have no rows nowhere."""
    import ctypes

    import torch
    lr = ExtRun(*CASES["d64_gqa4_buffers"])
    L = _lib.lib()

    def count(name):
        ms, n = ctypes.c_double(), ctypes.c_int64()
        _lib.check(L.seg_profile_read(name.encode(), ctypes.byref(ms), ctypes.byref(n)))
        return n.value
    L.seg_profile_reset()
    L.seg_profile_enable(1)
    try:
        s8 = S.layer_saved8(lr.lay, lr.lc, True)
        S.seg_layer_fwd_ext(lr.lay, lr.lc, lr.w, lr.x, lr.rope, lr.pos, saved8=s8)
        assert count("ly_act8") >= 1 and count("act_pack") == 0
        S.seg_layer_bwd_ext(lr.lay, lr.lc, lr.w, lr.dy, lr.rope, lr.pos, saved8=s8)
        assert count("ly_act8") >= 2 and count("act_unpack") == count("act_pack") == 0
        S.seg_act_pack(S.seg_act_unpack(s8["x"]))
        x = torch.ones(4, 32, device=lr.dev)
        with pytest.raises(_lib.SegError):
            S.seg_act_pack(x, S.Act8(x.view(torch.int8).flatten()[:128].view(4, 32), s8["x"].exp[:4, :1].contiguous()))
        S.seg_act_pack(x[:0])
        assert count("act_unpack") == count("act_pack") == 1
    finally:
        L.seg_profile_enable(0)
        L.seg_profile_reset()


@pytest.mark.parametrize("keep_gate", [False, True])
@pytest.mark.parametrize("x_by,k_by", [(32, 1), (1, 16), (32, 16)])
def test_large_channels(x_by, k_by, keep_gate):
    """A few channels of the residual stream 32 times (with norm weights 1 / 32 there), and two of
    every key head 16 times the others, which leaves their blocks' other columns two or three bits.
    The backward equals that of the kept values in 64 bits (probabilities against the forward's
    lse) within the bound of bf16 results; next to the gradients in bf16 it is off by what 64
    bits give for the format alone, E, and the two calls' own bounds."""
    import torch
    say(x_by, k_by, keep_gate)
    lr = ExtRun(*CASES["d128_chunked"])
    c, ch = lr.cfg, [5, 77, 200]
    x, w, ref, masks, a, dy = lr.oracle_parts()
    key = [h * c.head_dim + i for h in range(c.hkv) for i in (3, 70)]
    for t in (x, lr.x):
        t[:, ch] *= x_by
    for n, rows, by in (("g1", ch, 1 / x_by), ("g2", ch, 1 / x_by), ("wk", key, k_by)):
        lr.w[n][rows] *= by
        getattr(w, n)[rows] *= by
    y, saved = S.seg_layer_fwd_ext(lr.lay, lr.lc, lr.w, lr.x, lr.rope, lr.pos)
    dx16, g16 = S.seg_layer_bwd_ext(lr.lay, lr.lc, lr.w, lr.dy, lr.rope, lr.pos, x=lr.x, saved=saved)
    s8 = S.layer_saved8(lr.lay, lr.lc, keep_gate)
    S.seg_layer_fwd_ext(lr.lay, lr.lc, lr.w, lr.x, lr.rope, lr.pos, saved8=s8)
    dx, grads = S.seg_layer_bwd_ext(lr.lay, lr.lc, lr.w, lr.dy, lr.rope, lr.pos, saved8=s8)
    ok = ref.tok_src >= 0

    def backward(x8, sv):
        """from kept values: both norms' and the block's of x and y1, unless g and u are kept"""
        sv["a"], _ = OLY.rms_forward(x8, w.g1, EPS)
        sv["b"], _ = OLY.rms_forward(sv["y1"], w.g2, EPS)
        if "gt" not in sv:
            sv["gt"], sv["ut"] = sv["b"] @ w.wg.T, sv["b"] @ w.wu.T
        sv["mm"] = OLY.silu(sv["gt"]) * sv["ut"]
        return OLY.backward(x8, w, ref.segments, masks, **a, saved=sv, dy=dy, own_softmax=False)

    def values(t, *shape):
        t = _np(t)
        t[~ok] = 0
        return t.reshape(lr.P, *shape) if shape else t
    heads = {"q": (c.hq, c.head_dim), "k": (c.hkv, c.head_dim), "v": (c.hkv, c.head_dim), "o": (c.hq, c.head_dim)}
    sv = {n + ("r" if n in "qk" else ""): values(S.seg_act_unpack(s8[n]), *shape) for n, shape in heads.items()}
    sv.update(y1=values(S.seg_act_unpack(s8["y1"])), lse=_np(s8["lse"]), pos=OLY.segment_positions(ref.segments, lr.P))
    sv["r1"], sv["r2"] = (np.where(ok, _np(s8[n]), 0) for n in ("rstd1", "rstd2"))
    if keep_gate:
        sv["gt"], sv["ut"] = (values(S.seg_act_unpack(s8[n])) for n in ("g", "u"))
    want = backward(values(S.seg_act_unpack(s8["x"])), sv)
    # the format alone: 64-bit values packed
    _, ex = OLY.forward(x, w, ref.segments, masks, **a)
    full = OLY.backward(x, w, ref.segments, masks, **a, saved=ex, dy=dy)

    def keep(t):
        return OA8.unpack(*OA8.pack(t.reshape(lr.P, -1))).reshape(t.shape)
    packed = {n: keep(ex[n]) if n in ("qr", "kr", "v", "o", "y1") or keep_gate and n in ("gt", "ut") else ex[n]
              for n in ex if keep_gate or n not in ("gt", "ut")}
    alone = backward(keep(x), packed)
    named = lambda r: {"dx": np.where(ok[:, None], r[0], 0), **r[1]}  # noqa: E731
    want, full, alone = named(want), named(full), named(alone)
    for n, got in {"dx": dx, **grads}.items():
        E = rel(alone[n], full[n])
        d16 = rel(_np(got), _np(dx16 if n == "dx" else g16[n]))
        say(n, f"of the kept values {rel(_np(got), want[n]):.4f}, next to bf16 {d16:.4f}, the format {E:.4f}")
        assert rel(_np(got), want[n]) < TOL, n
        assert d16 < E + 2 * TOL, n
