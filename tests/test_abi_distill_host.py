"""Host-side checks of the operators of a teacher and its student (no GPU): structures,
workspace sizes, and what each entry point refuses before any launch."""
import ctypes

import pytest

from paper_2607_11185_amd import _lib
from paper_2607_11185_amd import seg as S
from tests.test_abi_host import _lib_or_skip
from tests import test_abi_structs as TS

ARG, CAP, WS, UNS = (_lib.SEG_ERR_ARG, _lib.SEG_ERR_CAPACITY, _lib.SEG_ERR_WORKSPACE, _lib.SEG_ERR_UNSUPPORTED)
STRUCTS = {"seg_fp8": _lib.SegFp8, "seg_distill_cfg": _lib.SegDistillCfg}
MB = 1 << 20


def test_structures_match_header(tmp_path, monkeypatch):
    monkeypatch.setattr(TS, "STRUCTS", STRUCTS)
    TS.test_ctypes_structs_match_header(tmp_path)
    TS.test_header_fields_all_mirrored()


@pytest.mark.parametrize("kw,want", [
    (dict(rows=-1), ARG), (dict(cols=0), ARG), (dict(ldx=63), ARG), (dict(dt=5), UNS), (dict(x=None), ARG), (dict(p=None), ARG),
    (dict(code=None), ARG), (dict(exp=None), ARG), (dict(x=17), ARG), (dict(x=18, dt=1), ARG), (dict(rows=1 << 41), CAP),
    (dict(rows=1 << 35, cols=1 << 20, ldx=1 << 20), CAP), (dict(rows=1 << 34), CAP), (dict(block_rows=0), UNS),
    (dict(block_rows=64), UNS), (dict(block_rows=-1), UNS), (dict(code=MB + 8), UNS), (dict(exp=2 * MB + 4), UNS)])
def test_packing_refuses(kw, want):
    L = _lib_or_skip()
    a = dict(rows=4, cols=64, ldx=64, dt=0, x=16, p=True, code=MB, exp=2 * MB, block_rows=1)
    a.update(kw)
    s = _lib.SegFp8(a["code"], a["exp"], a["block_rows"])
    p = ctypes.byref(s) if a["p"] else None
    assert L.seg_fp8_pack(a["rows"], a["cols"], a["dt"], a["x"], a["ldx"], p, None) == want
    assert L.seg_last_error()
    assert L.seg_fp8_unpack(a["rows"], a["cols"], a["dt"], p, a["x"], a["ldx"], None) == want


@pytest.mark.parametrize("x,code,exp", [(16, 16, MB), (16, MB, 16), (16, MB, 512), (MB, 16, 256), (4096, 256, 256 + 240), (256, 16, MB)])
def test_packing_refuses_overlapping_arrays(x, code, exp):
    """4 rows of 64 columns: 512 bytes of x, 256 of codes, 16 of exponents."""
    L = _lib_or_skip()
    s = _lib.SegFp8(code, exp, 1)
    assert L.seg_fp8_pack(4, 64, 0, x, 64, ctypes.byref(s), None) == ARG


def _gemm(rows=100, outs=40, cols=8192, dt=0, y=MB, ldy=40, ws=8 * MB, ws_bytes=1 << 40, a=(16 * MB, 32 * MB, 1),
          b=(48 * MB, 64 * MB, 128)):
    L = _lib_or_skip()
    sa, sb = (None if v is None else ctypes.byref(_lib.SegFp8(*v)) for v in (a, b))
    return L.seg_fp8_gemm(rows, outs, cols, sa, sb, dt, y, ldy, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,want", [
    (dict(dt=2), UNS), (dict(rows=-1), ARG), (dict(outs=0), ARG), (dict(cols=0), ARG), (dict(rows=(1 << 20) + 1), CAP),
    (dict(outs=(1 << 20) + 1, ldy=2 << 20), CAP), (dict(cols=(1 << 20) + 1), CAP), (dict(ldy=39), ARG), (dict(a=None), ARG), (dict(b=None), ARG),
    (dict(a=(None, 32 * MB, 1)), ARG), (dict(b=(48 * MB, None, 128)), ARG), (dict(a=(16 * MB + 8, 32 * MB, 1)), UNS),
    (dict(b=(48 * MB, 64 * MB + 1, 128)), UNS), (dict(b=(48 * MB, 64 * MB, 32)), UNS), (dict(ws_bytes=100), WS), (dict(ws=None), ARG),
    (dict(ws=8 * MB + 4), UNS), (dict(y=None), ARG), (dict(y=MB + 1), ARG), (dict(y=MB + 2, dt=1), ARG),
    (dict(y=16 * MB), ARG), (dict(y=32 * MB), ARG), (dict(y=48 * MB), ARG), (dict(y=64 * MB), ARG), (dict(y=8 * MB), ARG),
    (dict(ws=16 * MB - 16), ARG), (dict(ws=MB), ARG), (dict(a=(MB, 32 * MB, 1)), ARG)])
def test_product_refuses(kw, want):
    assert _gemm(**kw) == want
    assert _lib.lib().seg_last_error()


def test_product_of_nothing_and_sizes():
    L = _lib_or_skip()
    assert _gemm(rows=0, a=None, b=None, y=None, ws=None, ws_bytes=0) == _lib.SEG_OK
    for bad in ((-1, 4, 4), (4, 0, 4), (4, 4, 0), ((1 << 20) + 1, 4, 4)):
        assert L.seg_fp8_gemm_workspace_bytes(*bad) == 0
    assert L.seg_fp8_gemm_workspace_bytes(64, 40, 8192) == 0      # few rows need none
    assert L.seg_fp8_gemm_workspace_bytes(100, 40, 8192) % (100 * 48 * 4) < 256


def test_binding_refuses():
    import torch
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        S.seg_fp8_pack(x, 64)
    with pytest.raises(TypeError):
        S.seg_fp8_pack(x.half())
    with pytest.raises(AssertionError):                            # not on a GPU
        S.seg_fp8_pack(x)
    with pytest.raises(AssertionError):
        S.seg_fp8_pack(x, 1, S.Fp8.empty(4, 65, 1, "cpu"))
    with pytest.raises(AssertionError):
        S.seg_fp8_pack(x, 128, S.Fp8.empty(4, 64, 1, "cpu"))
    a, b = S.Fp8.empty(4, 64, 1, "cpu"), S.Fp8.empty(5, 65, 128, "cpu")
    with pytest.raises(AssertionError):                            # other columns
        S.seg_fp8_gemm(a, b)
    bad = S.Fp8(a.code, a.exp[:, :8], 64, 1)
    with pytest.raises(AssertionError):
        bad.c()


# ---------------------------------------------------------------- top logits

def _top(rows=4, vocab=5000, k=10, dt=0, z=MB, ldz=5000, scale=1.0, ids=2 * MB, logits=3 * MB, lse=4 * MB, ws=8 * MB,
         ws_bytes=1 << 40):
    return _lib_or_skip().seg_top_logits(rows, vocab, k, dt, z, ldz, scale, ids, logits, lse, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,want", [
    (dict(dt=2), UNS), (dict(rows=-1), ARG), (dict(vocab=0), ARG), (dict(k=0), ARG), (dict(k=5001), ARG), (dict(k=257), UNS),
    (dict(vocab=(1 << 20) + 1, ldz=2 << 20), CAP), (dict(rows=(1 << 20) + 1), CAP), (dict(ldz=4999), ARG),
    (dict(scale=float("nan")), ARG), (dict(scale=float("inf")), ARG), (dict(ws_bytes=100), WS), (dict(z=None), ARG), (dict(ids=None), ARG),
    (dict(logits=None), ARG), (dict(lse=None), ARG), (dict(ws=None), ARG), (dict(z=MB + 1), ARG), (dict(z=MB + 2, dt=1), ARG),
    (dict(ws=8 * MB + 8), UNS), (dict(ids=MB + 7996), ARG), (dict(lse=3 * MB + 156), ARG), (dict(logits=8 * MB), ARG),
    (dict(ws=MB + 4096), ARG), (dict(rows=1 << 20, vocab=1 << 20, ldz=1 << 20, z=1 << 44), CAP)])
def test_top_logits_refuse(kw, want):
    assert _top(**kw) == want
    assert _lib.lib().seg_last_error()


def test_top_logits_of_nothing_and_sizes():
    L = _lib_or_skip()
    assert _top(rows=0, z=None, ids=None, logits=None, lse=None, ws=None, ws_bytes=0) == _lib.SEG_OK
    for bad in ((-1, 4), (4, 0), ((1 << 20) + 1, 4), (4, (1 << 20) + 1)):
        assert L.seg_top_logits_workspace_bytes(*bad) == 0
    assert L.seg_top_logits_workspace_bytes(4, 5000) > 0 and L.seg_top_logits_workspace_bytes(511, 151936) > 0
    # one kernel, no workspace: small vocabularies and many rows
    assert L.seg_top_logits_workspace_bytes(4, 4096) == L.seg_top_logits_workspace_bytes(512, 151936) == 0


# -------------------------------------------------------------- distillation

def _distill(rows=40, hidden=64, vocab=1000, k=10, dt=0, n_h=40, h=MB, row_index=None, w=2 * MB, ids=3 * MB, logits=4 * MB,
             t_lse=None, weight=None, cfg=(1.0, 1.0, 1.0, 1), loss_tok=5 * MB, lse=6 * MB, loss_sum=7 * MB, dh=8 * MB, dw_dt=0,
             dw=9 * MB, ws=64 * MB, ws_bytes=1 << 40):
    c = None if cfg is None else ctypes.byref(_lib.SegDistillCfg(*cfg))
    return _lib_or_skip().seg_distill_loss(rows, hidden, vocab, k, dt, n_h, h, row_index, w, ids, logits, t_lse, weight, c, loss_tok,
                                           lse, loss_sum, dh, dw_dt, dw, ws, ws_bytes, None)


INF = float("inf")


@pytest.mark.parametrize("kw,want", [
    (dict(cfg=None), ARG), (dict(dt=2), ARG), (dict(dw_dt=2), ARG), (dict(rows=-1), ARG), (dict(hidden=0), ARG), (dict(vocab=0), ARG),
    (dict(n_h=-1), ARG), (dict(k=0), ARG), (dict(k=1001), ARG), (dict(k=257), UNS), (dict(hidden=60), UNS), (dict(rows=1 << 20, n_h=1 << 20), CAP),
    (dict(vocab=1 << 20), CAP), (dict(hidden=(1 << 20) + 8), CAP), (dict(cfg=(INF, 1, 1, 1)), ARG), (dict(cfg=(1, float("nan"), 1, 1)), ARG),
    (dict(cfg=(1, 1, -INF, 1)), ARG), (dict(n_h=39), ARG), (dict(ws_bytes=1000), WS), (dict(h=None), ARG), (dict(w=None), ARG),
    (dict(ids=None), ARG), (dict(logits=None), ARG), (dict(loss_tok=None), ARG), (dict(lse=None), ARG), (dict(loss_sum=None), ARG),
    (dict(dh=None), ARG), (dict(dw=None), ARG), (dict(ws=None), ARG), (dict(h=MB + 1), ARG), (dict(dh=8 * MB + 1), ARG), (dict(dw=9 * MB + 2, dw_dt=1), ARG),
    (dict(w=2 * MB + 8), UNS), (dict(ws=64 * MB + 8), UNS), (dict(dw=2 * MB), ARG), (dict(dh=MB + 5118), ARG), (dict(loss_tok=3 * MB), ARG),
    (dict(lse=5 * MB + 156), ARG), (dict(loss_sum=4 * MB), ARG), (dict(ws=9 * MB), ARG), (dict(dh=9 * MB), ARG), (dict(t_lse=6 * MB), ARG),
    (dict(weight=5 * MB), ARG), (dict(row_index=8 * MB), ARG)])
def test_distillation_refuses(kw, want):
    assert _distill(**kw) == want
    assert _lib.lib().seg_last_error()


def test_distillation_sizes():
    L = _lib_or_skip()
    for bad in ((-1, 64, 1000, 10), (4, 0, 1000, 10), (4, 64, 0, 10), (4, 64, 1000, 0), (4, 64, 1000, 257), (1 << 20, 64, 1000, 10)):
        assert L.seg_distill_workspace_bytes(*bad, 0, 1) == 0
    a, b = (L.seg_distill_workspace_bytes(40, 64, 1000, 10, 0, g) for g in (0, 1))
    assert 0 < a < b < L.seg_distill_workspace_bytes(40, 64, 1000, 10, 1, 1)
    assert _distill(rows=0, n_h=0, dw=None) == ARG and _distill(ws_bytes=b - 1) == WS


def test_distillation_binding_refuses():
    import torch
    h, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(30, 64, dtype=torch.bfloat16)
    ids, logits = torch.zeros(4, 5, dtype=torch.int32), torch.zeros(4, 5)
    good = dict(h=h, row_index=None, w=w, ids=ids, logits=logits, cfg=S.DistillCfg())
    for bad in (dict(w=w[:, :32]), dict(w=w.float()), dict(ids=ids.long()), dict(logits=logits[:, :4]), dict(logits=logits.double()),
                dict(row_index=torch.zeros(4, dtype=torch.int64)), dict(row_index=torch.zeros(3, dtype=torch.int32)),
                dict(t_lse=torch.zeros(3)), dict(row_weight=torch.zeros(4, 1)), dict(dw_dtype=torch.float16), dict()):
        with pytest.raises((AssertionError, TypeError)):
            S.seg_distill_loss(**{**good, **bad})


@pytest.mark.parametrize("rows,cols,block_rows,pack,unpack", [
    # 2^23 thread blocks of 16 rows, and one more; overlapping arrays are refused behind the size
    (1 << 27, 1, 1, ARG, ARG), ((1 << 27) + 1, 1, 1, CAP, CAP),
    # of 128 rows: their own grid when they are packed
    (1, 1 << 30, 128, ARG, ARG), (128, 1 << 30, 128, ARG, CAP), (129, 1 << 30, 128, CAP, CAP), (1 << 30, 1, 128, ARG, CAP),
    ((1 << 30) + 1, 1, 128, CAP, CAP)])
def test_packing_is_bounded_by_its_own_grid(rows, cols, block_rows, pack, unpack):
    L = _lib_or_skip()
    s = _lib.SegFp8(256, 1 << 50, block_rows)
    assert L.seg_fp8_pack(rows, cols, 0, 256, cols, ctypes.byref(s), None) == pack
    assert L.seg_fp8_unpack(rows, cols, 0, ctypes.byref(s), 256, cols, None) == unpack


@pytest.mark.parametrize("rows,vocab,want", [(1 << 20, 131072, ARG), (1 << 20, 262144, ARG), (1 << 20, 262145, CAP), (1 << 18, 524289, CAP),
                                             ((1 << 18) - 1, 524288, ARG)])
def test_top_logits_are_bounded_by_what_is_launched(rows, vocab, want):
    """Parts of 16,384 columns a block, 2^23 - 1 of them, unless a block takes a row; an output
    on the logits is refused behind that."""
    assert _top(rows=rows, vocab=vocab, ldz=vocab, z=1 << 30, ids=1 << 31, ws=1 << 60, logits=1 << 61, lse=1 << 59, ws_bytes=1 << 50) == want


def test_forward_alone_does_not_look_at_gradients():
    """Misaligned dh and dw go unnoticed without want_grad (w's own check is behind theirs)."""
    kw = dict(dh=8 * MB + 1, dw=9 * MB + 2, dw_dt=1, w=2 * MB + 8)
    assert _distill(cfg=(1.0, 1.0, 1.0, 0), **kw) == UNS
    assert _distill(**kw) == ARG
