"""Host-side checks of the three-axis positions, the rotation, the 8-bit
activations and the gated block (no GPU): structures, workspace sizes, and
what each entry point refuses before any launch."""
import ctypes

import numpy as np
import pytest

from paper_2607_11185_amd import _lib
from paper_2607_11185_amd import seg as S
from paper_2607_11185_amd import workload as WL
from tests.test_abi_host import _lib_or_skip, _prob
from tests import test_abi_structs as TS

ARG, CAP, WS, UNS = (_lib.SEG_ERR_ARG, _lib.SEG_ERR_CAPACITY, _lib.SEG_ERR_WORKSPACE, _lib.SEG_ERR_UNSUPPORTED)
STRUCTS = {"seg_mrope_cfg": _lib.SegMropeCfg, "seg_act8": _lib.SegAct8, "seg_layer_saved8": _lib.SegLayerSaved8,
           "seg_layer_ext": _lib.SegLayerExt}


def test_structures_match_header(tmp_path, monkeypatch):
    monkeypatch.setattr(TS, "STRUCTS", STRUCTS)
    TS.test_ctypes_structs_match_header(tmp_path)
    TS.test_header_fields_all_mirrored()


def _positions(pr, grid, sz=None, ws_bytes=1 << 30, pos=None, ws=None):
    L = _lib_or_skip()
    sz = sz or S.seg_layout_query(pr)
    g = None if grid is None else np.ascontiguousarray(grid, np.int32)
    return L.seg_mrope_positions(ctypes.byref(pr.c()), ctypes.byref(sz), None if g is None else g.ctypes.data, pos, ws,
                                 ws_bytes, None)


GOOD = [[1, 5, 1, 1], [1, 1, 5, 0], [5, 1, 1, 2]]


@pytest.mark.parametrize("step,row,want", [
    (0, [1, 2, 2, 1], ARG),            # four patches for five tokens
    (1, [0, 5, 1, 1], ARG), (1, [-1, -5, 1, 1], ARG), (2, [1, -1, -5, 1], ARG),
    (2, [5, 1, 1, -1], ARG),           # negative time step
    (0, [2 ** 30, 2 ** 30, 2 ** 30, 1], ARG), (0, [65536, 65536, 5, 1], ARG),
    (2, [5, 1, 1, 2 ** 30], CAP)])     # four steps of 2^30 positions
def test_positions_refuse_bad_grids(step, row, want):
    pr = _prob()
    L = _lib_or_skip()
    grid = [list(g) for g in GOOD]
    grid[step] = row
    assert _positions(pr, grid) == want
    assert L.seg_last_error()


def test_positions_refuse_bad_calls():
    L = _lib_or_skip()
    pr = _prob()
    sz = S.seg_layout_query(pr)
    assert L.seg_mrope_positions_workspace_bytes(ctypes.byref(pr.c()), ctypes.byref(sz)) > 0
    assert _positions(pr, None) == ARG and b"grid" in L.seg_last_error()
    assert _positions(pr, GOOD, ws_bytes=255) == WS
    assert _positions(pr, GOOD) == ARG and b"NULL" in L.seg_last_error()       # pos and ws
    other = _lib.SegSizes.from_buffer_copy(sz)
    other.packed_tokens += 1
    assert _positions(pr, GOOD, sz=other) == ARG
    assert L.seg_mrope_positions(None, ctypes.byref(sz), None, None, None, 0, None) == ARG
    assert L.seg_mrope_positions(ctypes.byref(pr.c()), None, None, None, None, 0, None) == ARG
    assert L.seg_mrope_positions_workspace_bytes(None, ctypes.byref(sz)) == 0
    assert L.seg_mrope_positions_workspace_bytes(ctypes.byref(pr.c()), None) == 0
    # the size that is asked for is enough, for any problem
    rng = np.random.default_rng(3)
    for _ in range(20):
        T = rng.integers(0, 30, size=3)
        n = int(T.sum())
        sp = WL.explicit_spans(T, rng.integers(1, 5, size=3), rng.integers(0, 2, size=n) * 6, rng.integers(0, 4, size=n), [0] * n)
        many = S.Problem.from_spans(sp, int(rng.integers(1, 9)), int(rng.integers(1, 5)), 0, int(rng.choice([0, 4000])))
        msz = S.seg_layout_query(many)
        size = L.seg_mrope_positions_workspace_bytes(ctypes.byref(many.c()), ctypes.byref(msz))
        grid = np.tile(np.array([1, 2, 3, 1], np.int32), (n, 1))
        assert _positions(many, grid, ws_bytes=size) == (ARG if msz.packed_tokens else _lib.SEG_OK)   # pos is NULL
    # a problem without screenshots needs no grid, and one without trajectories no memory
    text = S.Problem.from_spans(WL.explicit_spans([2], [3], [0, 0], [4, 4], [1, 1]), 1, 1)
    assert _positions(text, None) == ARG and b"pos or ws" in L.seg_last_error()
    none = S.Problem.from_spans(WL.explicit_spans([], [], [], [], []), 1, 1)
    assert _positions(none, None) == _lib.SEG_OK


def _rope(rows=4, dt=0, sections=(8, 12, 12), base=1e4, hq=2, hkv=1, d=64, pos=16, q=16, ldq=128, k=16, ldk=64,
          qo=16, ldqo=128, ko=16, ldko=64, cfg=True):
    L = _lib_or_skip()
    c = _lib.SegMropeCfg((ctypes.c_int32 * 3)(*sections), base)
    args = (rows, dt, ctypes.byref(c) if cfg else None, hq, hkv, d, pos, q, ldq, k, ldk, qo, ldqo, ko, ldko, None)
    got = L.seg_mrope_fwd(*args), L.seg_mrope_bwd(*args)
    assert got[0] == got[1]
    return got[0]


@pytest.mark.parametrize("kw,want", [
    (dict(cfg=False), ARG), (dict(rows=-1), ARG), (dict(rows=2 ** 31), CAP), (dict(dt=2), UNS),
    (dict(sections=(8, 12, 11)), ARG), (dict(sections=(-8, 20, 20)), ARG), (dict(sections=(2 ** 31 - 1, 2 ** 31 - 1, 34)), ARG),
    (dict(base=1.0), ARG), (dict(base=float("nan")), ARG), (dict(base=float("inf")), ARG),
    (dict(d=72, sections=(36, 0, 0)), UNS), (dict(d=0, sections=(0, 0, 0)), UNS), (dict(d=272, sections=(136, 0, 0)), UNS),
    (dict(hq=0), ARG), (dict(hkv=-1), ARG), (dict(hq=1 << 20), ARG),
    (dict(pos=None), ARG), (dict(q=None), ARG), (dict(k=None), ARG), (dict(qo=None), ARG), (dict(ko=None), ARG),
    (dict(ldq=127), ARG), (dict(ldk=32), ARG), (dict(ldqo=64), ARG), (dict(ldq=132), UNS), (dict(q=20), UNS), (dict(ko=8), UNS)])
def test_rotation_refuses(kw, want):
    assert _rope(**kw) == want


@pytest.mark.parametrize("kw", [
    dict(qo=1 << 20, ldqo=136), dict(qo=(1 << 20) + 16), dict(qo=(1 << 20) + 256), dict(qo=(1 << 20) - 16), dict(ko=2 << 20, ldko=72),
    dict(ko=1 << 20), dict(qo=2 << 20), dict(qo=4 << 20), dict(ko=(3 << 20) + 3 * 256 + 240),
    # parts of one wide row: the next one's columns, its own of another row, its last columns
    dict(ldq=256, ldqo=256, qo=(1 << 20) + 240), dict(ldq=256, ldqo=256, qo=(1 << 20) + 512),
    dict(ldq=256, ldqo=256, qo=(1 << 20) + 272), dict(rows=1, qo=(1 << 20) + 240)])
def test_rotation_refuses_overlapping_tensors(kw):
    """An output on an input that is not its own, or at another stride or offset of its own."""
    assert _rope(**dict(dict(q=1 << 20, k=2 << 20, qo=3 << 20, ko=4 << 20), **kw)) == ARG


def test_rotation_of_nothing():
    assert _rope(rows=0, pos=None, q=None, k=None, qo=None, ko=None) == _lib.SEG_OK


@pytest.mark.parametrize("kw,want", [
    (dict(rows=-1), ARG), (dict(cols=0), ARG), (dict(ldx=63), ARG), (dict(dt=5), UNS), (dict(x=None), ARG), (dict(p=None), ARG),
    (dict(code=None), ARG), (dict(exp=None), ARG), (dict(x=17), ARG), (dict(x=18, dt=1), ARG), (dict(rows=1 << 41), CAP),
    (dict(rows=1 << 39, cols=1 << 20, ldx=1 << 20), CAP), (dict(rows=1 << 36), CAP)])
def test_packing_refuses(kw, want):
    L = _lib_or_skip()
    a = dict(rows=4, cols=64, ldx=64, dt=0, x=16, p=True, code=8, exp=1)
    a.update(kw)
    s = _lib.SegAct8(a["code"], a["exp"])
    p = ctypes.byref(s) if a["p"] else None
    assert L.seg_act_pack(a["rows"], a["cols"], a["dt"], a["x"], a["ldx"], p, None) == want
    assert L.seg_act_unpack(a["rows"], a["cols"], a["dt"], p, a["x"], a["ldx"], None) == want


@pytest.mark.parametrize("x,code,exp", [(16, 16, 1 << 20), (16, 1 << 20, 16 + 510), (1 << 20, 16, 16 + 255), (256, 1, 1 << 20)])
def test_packing_refuses_overlapping_arrays(x, code, exp):
    L = _lib_or_skip()
    s = _lib.SegAct8(code, exp)
    assert L.seg_act_pack(4, 64, 0, x, 64, ctypes.byref(s), None) == ARG
    assert L.seg_act_unpack(4, 64, 0, ctypes.byref(s), x, 64, None) == ARG


def test_packing_of_nothing():
    L = _lib_or_skip()
    s = _lib.SegAct8(None, None)
    assert L.seg_act_pack(0, 64, 0, None, 64, ctypes.byref(s), None) == _lib.SEG_OK
    assert L.seg_act_unpack(0, 64, 0, ctypes.byref(s), None, 64, None) == _lib.SEG_OK


@pytest.mark.parametrize("kw,want", [
    (dict(rows=-1), ARG), (dict(rows=(1 << 20) + 1), UNS), (dict(hidden=60), UNS), (dict(inter=100), UNS), (dict(hidden=0), UNS),
    (dict(inter=(1 << 20) + 8), UNS), (dict(rows=1 << 20, inter=1 << 19), CAP), (dict(hidden=1 << 19, ldx=1 << 19, inter=1 << 20), CAP),
    (dict(ldx=56), ARG), (dict(ldx=68), UNS), (dict(x=None), ARG), (dict(wu=None), ARG),
    (dict(x=8), UNS), (dict(wg=24), UNS), (dict(u8=False), ARG), (dict(g8=False), ARG), (dict(code=None), ARG), (dict(code=4), UNS)])
def test_gated_block_refuses(kw, want):
    L = _lib_or_skip()
    a = dict(rows=4, hidden=64, inter=96, ldx=64, x=16, wg=16, wu=16, g8=True, u8=True, code=8)
    a.update(kw)
    s = _lib.SegAct8(a["code"], 1)
    g8, u8 = (ctypes.byref(s) if a[n] else None for n in ("g8", "u8"))
    size = (a["rows"], a["hidden"], a["inter"], a["x"], a["ldx"], a["wg"], a["wu"])
    assert L.seg_glu_fwd(*size, 16, g8, u8, 16, 1 << 40, None) == want
    assert L.seg_glu_bwd(*size, g8, u8, 16, 16, 16, 0, 16, 16, 16, 1 << 40, None) == want


def test_gated_block_backward_refuses():
    L = _lib_or_skip()
    size = (4, 64, 96, 16, 64, 16, 16)
    need = L.seg_glu_workspace_bytes(4, 64, 96, 1, 0)
    kept = L.seg_glu_workspace_bytes(4, 64, 96, 1, 1)
    fwd = L.seg_glu_workspace_bytes(4, 64, 96, 0, 0)
    assert 0 < fwd < kept < need and L.seg_glu_workspace_bytes(-1, 64, 96, 1, 1) == 0
    assert L.seg_glu_workspace_bytes((1 << 20) + 1, 64, 96, 0, 0) == 0
    s = _lib.SegAct8(8, 1)
    g = ctypes.byref(s)

    def bwd(g8=None, dm=16, m=16, dx=16, dt=0, dwg=16, dwu=16, ws=16, n=1 << 40):
        return L.seg_glu_bwd(*size, g8, g8, dm, m, dx, dt, dwg, dwu, ws, n, None)
    assert bwd(n=need - 1) == WS and bwd(g8=g, n=kept - 1) == WS
    assert bwd(dm=None) == bwd(dx=None) == bwd(dwg=None) == bwd(dwu=None) == bwd(ws=None) == ARG
    assert bwd(dm=8) == bwd(m=8) == bwd(dx=8) == bwd(dwg=8) == bwd(dwu=8) == bwd(ws=8) == bwd(dt=3) == UNS
    assert L.seg_glu_fwd(*size, None, None, None, 16, fwd, None) == ARG
    assert L.seg_glu_fwd(*size, 16, None, None, 16, fwd - 1, None) == WS
    assert L.seg_glu_fwd(*size, 16, None, None, None, fwd, None) == ARG
    assert L.seg_glu_fwd(*size, 16, None, None, 8, fwd, None) == UNS
    assert L.seg_glu_fwd(0, 64, 96, None, 64, None, None, None, None, None, None, 0, None) == _lib.SEG_OK


def test_gated_block_refuses_overlapping_tensors():
    """An output or the workspace on an input, or on another output: dx over x for one,
    which the weight gradients read afterwards."""
    L = _lib_or_skip()
    R, H, I = 4, 64, 96
    size = {"x": R * H * 2, "wg": I * H * 2, "wu": I * H * 2, "m": R * I * 2, "dm": R * I * 2, "dx": R * H * 2,
            "dwg": I * H * 4, "dwu": I * H * 4, "gc": R * I, "ge": R * 3, "uc": R * I, "ue": R * 3}
    need = {0: L.seg_glu_workspace_bytes(R, H, I, 0, 0), 1: L.seg_glu_workspace_bytes(R, H, I, 1, 1)}
    at, names = {}, {0: ["x", "wg", "wu", "m", "gc", "ge", "uc", "ue", "ws"],
                     1: ["x", "wg", "wu", "m", "gc", "ge", "uc", "ue", "dm", "dx", "dwg", "dwu", "ws"]}
    for i, n in enumerate([*size, "ws"]):
        at[n] = (i + 1) << 20

    def call(bwd, p):
        g8, u8 = ctypes.byref(_lib.SegAct8(p["gc"], p["ge"])), ctypes.byref(_lib.SegAct8(p["uc"], p["ue"]))
        if bwd:
            return L.seg_glu_bwd(R, H, I, p["x"], H, p["wg"], p["wu"], g8, u8, p["dm"], p["m"], p["dx"], 1, p["dwg"],
                                 p["dwu"], p["ws"], need[1], None)
        return L.seg_glu_fwd(R, H, I, p["x"], H, p["wg"], p["wu"], p["m"], g8, u8, p["ws"], need[0], None)
    for bwd in (0, 1):
        size["ws"] = need[bwd]
        outs = {"ws", "m", "dx", "dwg", "dwu"} if bwd else {"ws", "m", "gc", "ge", "uc", "ue"}
        for a in names[bwd]:
            for b in names[bwd]:
                if a != b and a in outs:
                    assert call(bwd, dict(at, **{a: at[b]})) == ARG, (bwd, a, b)
                    assert call(bwd, dict(at, **{a: at[b] + (size[b] - 1) // 16 * 16})) == ARG, (bwd, a, b)


def test_extended_layer_refuses():
    L = _lib_or_skip()
    sz = S.seg_layout_query(_prob())
    lay = _lib.SegLayout()
    lay.tile, lay.window = 128, 2
    cfg = S.LayerCfg(256, 512, 4, 2, 64).c()
    w = _lib.SegLayerWeights(*([1] * 9))
    g = _lib.SegLayerGrads(*([1] * 9))
    sv = _lib.SegLayerSaved(*([1] * 8))

    def size(saved8, bwd):
        return L.seg_layer_ext_workspace_bytes(ctypes.byref(sz), ctypes.byref(cfg), saved8, bwd)
    for bwd in (0, 1):
        assert size(0, bwd) == L.seg_layer_workspace_bytes(ctypes.byref(sz), ctypes.byref(cfg), bwd) < size(1, bwd)
    assert L.seg_layer_ext_workspace_bytes(None, ctypes.byref(cfg), 1, 0) == 0

    def both(e, want, saved=sv, x=1, n=1 << 40):
        e, saved = (None if v is None else ctypes.byref(v) for v in (e, saved))
        head = (ctypes.byref(lay), ctypes.byref(sz), ctypes.byref(cfg), e, ctypes.byref(w), x)
        assert L.seg_layer_fwd_ext(*head, 1, saved, 1, n, None) == want
        assert L.seg_layer_bwd_ext(*head, saved, 1, 1, ctypes.byref(g), 1, n, None) == want

    def ext(sections=(8, 12, 12), base=1e4, pos=1, drop=(), gate=True, code=8):
        e = _lib.SegLayerExt()
        if sections:
            e.rope = ctypes.pointer(_lib.SegMropeCfg((ctypes.c_int32 * 3)(*sections), base))
        e.pos = pos
        s = _lib.SegLayerSaved8()
        for n in _lib.SAVED8:
            if gate or n not in ("g", "u"):
                setattr(s, n, _lib.SegAct8(None if n in drop else code, None if n + ".exp" in drop else 1))
        for n in ("lse", "rstd1", "rstd2"):
            setattr(s, n, None if n in drop else 1)
        e.saved8 = ctypes.pointer(s)
        return e
    for bad in (dict(sections=(8, 12, 13)), dict(sections=(40, -4, -4)), dict(base=1.0), dict(pos=None), dict(drop=("g",)),
                dict(drop=("u",)), dict(drop=("u.exp",)), *(dict(drop=(n,)) for n in ("x", "q", "k", "v", "o", "y1", "lse", "rstd2")),
                dict(drop=("y1.exp",), gate=False)):
        both(ext(**bad), ARG)
    both(ext(code=4), UNS)
    both(ext(), WS, n=size(1, 0) - 1)
    both(ext(sections=None, gate=False), WS, n=size(1, 0) - 1)
    both(None, ARG, saved=None)              # nothing to save into
    both(_lib.SegLayerExt(), ARG, x=None)


def test_layer_binding_refuses():
    """Positions without their sections and base, saved vectors of another type, a layout
    on another device than the tensors."""
    import torch
    _lib_or_skip()
    sz = S.seg_layout_query(_prob())
    lay, cfg = S.Layout(sz, torch.device("cpu")), S.LayerCfg(256, 512, 4, 2, 64)
    P = sz.packed_tokens
    pos = torch.zeros(3, P, dtype=torch.int32)
    s8 = S.layer_saved8(lay, cfg)
    S._layer_ext(lay, cfg, S.MropeCfg((8, 12, 12)), pos, s8)
    for rope, p, saved in ((None, pos, None), (S.MropeCfg((8, 12, 12)), None, None),
                           (None, None, dict(s8, lse=s8["lse"].int())),
                           (None, None, dict(s8, rstd1=s8["rstd1"][:-1])),
                           (None, None, {n: v for n, v in s8.items() if n != "y1"})):
        with pytest.raises(AssertionError):
            S._layer_ext(lay, cfg, rope, p, saved)
    assert any(t is lay.tok_meta for t in S._layer_ext(lay, cfg, None, None, None)[1])


def test_extended_layer_refuses_overlapping_tensors():
    """With 8-bit saved activations an output, what is kept or the workspace on an input or on
    another of them is refused before any launch; y over x by an offset among them."""
    L = _lib_or_skip()
    sz = S.seg_layout_query(_prob())
    lay = _lib.SegLayout()
    lay.tile, lay.window = 128, 2
    H, I, hq, hkv, d, P = 256, 512, 4, 2, 64, sz.packed_tokens
    cfg = S.LayerCfg(H, I, hq, hkv, d).c()
    QD, KD = hq * d, hkv * d
    cols = {"x": H, "y1": H, "q": QD, "o": QD, "k": KD, "v": KD, "g": I, "u": I}
    kept = {f"{n}.{f}": P * (c if f == "code" else -(-c // 32)) for n, c in cols.items() for f in ("code", "exp")}
    kept.update(lse=hq * P * 4, rstd1=P * 4, rstd2=P * 4)
    weights = dict(zip(_lib.LAYER_WEIGHTS, (H, QD * H, KD * H, KD * H, H * QD, H, I * H, I * H, H * I)))
    acts = {"x": P * H * 2, "y": P * H * 2, "pos": 12 * P}
    size = {**kept, **{"w " + n: 2 * c for n, c in weights.items()}, **{"d " + n: 4 * c for n, c in weights.items()}, **acts}
    ws = [L.seg_layer_ext_workspace_bytes(ctypes.byref(sz), ctypes.byref(cfg), 1, b) for b in (0, 1)]
    at = {n: (i + 1) << 26 for i, n in enumerate(size)}
    at["ws"] = (len(at) + 1) << 26

    def call(bwd, p):
        e, s = _lib.SegLayerExt(), _lib.SegLayerSaved8()
        for n in cols:
            setattr(s, n, _lib.SegAct8(p[n + ".code"], p[n + ".exp"]))
        s.lse, s.rstd1, s.rstd2 = p["lse"], p["rstd1"], p["rstd2"]
        e.rope = ctypes.pointer(_lib.SegMropeCfg((ctypes.c_int32 * 3)(8, 12, 12), 1e4))
        e.pos, e.saved8 = p["pos"], ctypes.pointer(s)
        w = _lib.SegLayerWeights(*[p["w " + n] for n in _lib.LAYER_WEIGHTS])
        g = _lib.SegLayerGrads(*[p["d " + n] for n in _lib.LAYER_WEIGHTS])
        head = (ctypes.byref(lay), ctypes.byref(sz), ctypes.byref(cfg), ctypes.byref(e), ctypes.byref(w))
        if bwd:
            return L.seg_layer_bwd_ext(*head, None, None, p["x"], p["y"], ctypes.byref(g), p["ws"], ws[1], None)
        return L.seg_layer_fwd_ext(*head, p["x"], p["y"], None, p["ws"], ws[0], None)
    ins = [n for n in at if n.startswith("w ")] + ["x", "pos"]
    for bwd in (0, 1):
        size["ws"] = ws[bwd]
        outs = ["y", "ws", *([n for n in at if n.startswith("d ")] if bwd else kept)]
        others = ins + outs + (list(kept) if bwd else [])
        for a in outs:
            for b in others:
                if a == b or {a, b} == {"x", "y"}:
                    continue
                assert call(bwd, dict(at, **{a: at[b]})) == ARG, (bwd, a, b)
                assert call(bwd, dict(at, **{a: at[b] + size[b] - 1 if size[b] < 64 else at[b] + (size[b] - 1) // 16 * 16})) in (
                    (ARG, UNS) if a in ("g.code", "u.code") else (ARG,)), (bwd, a, b)
        for by in (16, H * 2, P * H * 2 - 16):
            assert call(bwd, dict(at, y=at["x"] + by)) == ARG and call(bwd, dict(at, y=at["x"] - by)) == ARG


def test_layer_backward_needs_what_the_forward_saved():
    """Without saved8 and without `saved` the binding allocates nothing to read from."""
    import torch
    _lib_or_skip()
    sz = S.seg_layout_query(_prob())
    lay, cfg = S.Layout(sz, torch.device("cpu")), S.LayerCfg(256, 512, 4, 2, 64)
    bf = dict(dtype=torch.bfloat16)
    shapes = dict(zip(_lib.LAYER_WEIGHTS, ((256,), (256, 256), (128, 256), (128, 256), (256, 256), (256,), (512, 256), (512, 256),
                                           (256, 512))))
    w = {n: torch.zeros(s, **bf) for n, s in shapes.items()}
    x = torch.zeros(sz.packed_tokens, 256, **bf)
    saved, _ = S._layer_saved(None, cfg, sz.packed_tokens, 256, x.device)
    for kw in (dict(x=x), dict(saved=saved), dict()):
        with pytest.raises(AssertionError, match="saved"):
            S.seg_layer_bwd_ext(lay, cfg, w, x, **kw)


@pytest.mark.parametrize("row", [0, 1, 3])
@pytest.mark.parametrize("out,width", [("qo", 256), ("ko", 128)])
def test_rotation_refuses_outputs_on_the_positions(out, width, row):
    """4 rows of `width` bytes, 512 bytes apart, and 48 bytes of positions that reach into a row's
    first or last byte or lie inside it."""
    base = 3 << 20
    kw = dict(q=1 << 20, k=2 << 20, qo=4 << 20, ko=5 << 20, ldqo=256, ldko=256)
    for at in (-47, -1, 0, 16, width - 1):
        assert _rope(**dict(kw, **{out: base, "pos": base + 512 * row + at})) == ARG
        assert b"pos" in _lib.lib().seg_last_error()


def test_positions_refuse_their_workspace():
    for pos, ws in ((1 << 20, 1 << 20), ((1 << 20) + 16, 1 << 20), (1 << 20, (1 << 20) + 16)):
        assert _positions(_prob(), GOOD, pos=pos, ws=ws) == ARG
