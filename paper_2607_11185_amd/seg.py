"""Python binding of the libseg entry points, on PyTorch device tensors.

Functions carry the C names (seg_layout_query, seg_build_layout, seg_attn_fwd,
seg_attn_bwd, seg_logprob_loss, seg_layer_fwd, seg_layer_bwd, seg_mrope_positions,
seg_mrope_fwd, seg_mrope_bwd, seg_act_pack, seg_act_unpack, seg_glu_fwd,
seg_glu_bwd, seg_layer_fwd_ext, seg_layer_bwd_ext, seg_fp8_pack, seg_fp8_unpack,
seg_fp8_gemm, seg_top_logits, seg_distill_loss) and only marshal arguments: they
allocate outputs and workspace with torch on the tensors' device and pass raw pointers
plus torch's current stream to the library.
"""
from __future__ import annotations

import contextlib
import ctypes
import dataclasses
from typing import Optional

import numpy as np

from . import _lib
from ._lib import SegLayout, SegLossCfg, SegProblem, SegSizes, check


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


@dataclasses.dataclass
class Problem:
    """Host-side problem (keeps the int32 span arrays alive for ctypes)."""
    step_offsets: np.ndarray
    prompt_len: np.ndarray
    img_len: np.ndarray
    text_len: np.ndarray
    action_len: np.ndarray
    window: int
    seg_steps: int
    max_seg_tokens: int = 0
    buffer_tokens: int = 0
    tile: int = 128
    mode: int = 0   # _lib.SEG_MODE_SLIDING or _lib.SEG_MODE_ANCHORED

    @classmethod
    def from_spans(cls, spans, window, seg_steps, max_seg_tokens=0, buffer_tokens=0, tile=128,
                   mode=0):
        if isinstance(mode, str):
            mode = {"sliding": _lib.SEG_MODE_SLIDING, "anchored": _lib.SEG_MODE_ANCHORED}[mode]
        return cls(_i32(spans.step_offsets), _i32(spans.prompt_len), _i32(spans.img_len),
                   _i32(spans.text_len), _i32(spans.action_len), int(window), int(seg_steps),
                   int(max_seg_tokens), int(buffer_tokens), int(tile), int(mode))

    def c(self) -> SegProblem:
        def ptr(a):
            return ctypes.cast(a.__array_interface__["data"][0] if a.size else None, _lib.P32)
        arrays = (self.step_offsets, self.prompt_len, self.img_len, self.text_len, self.action_len)
        p = SegProblem(len(self.prompt_len), *map(ptr, arrays), self.window, self.seg_steps,
                       self.max_seg_tokens, self.buffer_tokens, self.tile, self.mode)
        p.arrays = arrays  # alive as long as the struct
        return p


def seg_layout_query(problem: Problem) -> SegSizes:
    """Sizes of the layout (host only)."""
    sz = SegSizes()
    check(_lib.lib().seg_layout_query(ctypes.byref(problem.c()), ctypes.byref(sz)))
    return sz


def _stream(device) -> ctypes.c_void_p:
    import torch
    return ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


class Layout:
    """Device arrays of one layout (torch tensors) and the C struct over them."""

    FIELDS = ["seg_info", "tok_src", "tok_meta", "loss_pred_row", "loss_tgt_src", "loss_traj",
              "tile_seg", "qt_ptr", "qt_col", "qt_cls", "qt_ord", "kt_ptr", "kt_row", "kt_cls",
              "kt_ord", "seg_pairs", "tile_nnz"]

    def __init__(self, sizes: SegSizes, device):
        import torch
        S, P, R, G = (sizes.num_segments, sizes.packed_tokens, sizes.loss_rows, sizes.num_qtiles)
        Z = sizes.tile_nnz_max
        i32, u8, i64 = torch.int32, torch.uint8, torch.int64

        def e(n, dt):
            return torch.empty(max(int(n), 1), dtype=dt, device=device)

        self.sizes = sizes
        self.device = device
        self.seg_info = e(S * 8, i32)
        self.tok_src = e(P, i32)
        self.tok_meta = e(P, i32)
        self.loss_pred_row = e(R, i32)
        self.loss_tgt_src = e(R, i32)
        self.loss_traj = e(R, i32)
        self.tile_seg = e(G, i32)
        self.qt_ptr = e(G + 1, i32)
        self.qt_col = e(Z, i32)
        self.qt_cls = e(Z, u8)
        self.qt_ord = e(Z, i32)
        self.kt_ptr = e(G + 1, i32)
        self.kt_row = e(Z, i32)
        self.kt_cls = e(Z, u8)
        self.kt_ord = e(Z, i32)
        self.seg_pairs = e(S, i64)
        self.tile_nnz = e(1, i64)
        self.ws = e(sizes.workspace_bytes, u8)
        self.c = SegLayout(*[getattr(self, f).data_ptr() for f in self.FIELDS], 0, 0)

    def host(self) -> dict:
        """All arrays copied to host numpy, trimmed to their logical sizes."""
        s = self.sizes
        nnz = int(self.tile_nnz.cpu()[0]) if s.num_segments else 0
        lens = {"seg_info": s.num_segments * 8, "tok_src": s.packed_tokens,
                "tok_meta": s.packed_tokens, "loss_pred_row": s.loss_rows,
                "loss_tgt_src": s.loss_rows, "loss_traj": s.loss_rows,
                "tile_seg": s.num_qtiles, "qt_ptr": s.num_qtiles + 1, "qt_col": nnz,
                "qt_cls": nnz, "qt_ord": nnz, "kt_ptr": s.num_qtiles + 1, "kt_row": nnz,
                "kt_cls": nnz, "kt_ord": nnz, "seg_pairs": s.num_segments, "tile_nnz": 1}
        out = {f: getattr(self, f)[:lens[f]].cpu().numpy() for f in self.FIELDS}
        out["seg_info"] = out["seg_info"].reshape(-1, 8)
        out["xcd_rows"] = np.array(self.c.xcd_rows[:], np.int64)
        out["xcd_cols"] = np.array(self.c.xcd_cols[:], np.int64)
        return out


def seg_build_layout(problem: Problem, sizes: Optional[SegSizes] = None, device="cuda",
                     out: Optional[Layout] = None) -> Layout:
    """Build every layout array on the device.

    ``out`` reuses the arrays of an earlier layout of the same sizes.
    """
    import torch
    device = torch.device(device)
    if sizes is None:
        sizes = seg_layout_query(problem)
    if out is not None:
        if bytes(out.sizes) != bytes(sizes):
            raise ValueError("out was built for different sizes")
        lay = out
    else:
        lay = Layout(sizes, device)
    check(_lib.lib().seg_build_layout(ctypes.byref(problem.c()), ctypes.byref(sizes),
                                      ctypes.byref(lay.c), lay.ws.data_ptr(), lay.ws.numel(),
                                      _stream(device)))
    lay.window = problem.window
    return lay


def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.bfloat16:
        return _lib.SEG_BF16
    if t.dtype == torch.float32:
        return _lib.SEG_F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def attn_workspace(lay: Layout, dt: int, hq: int, hkv: int, d: int, bwd: bool):
    import torch
    n = _lib.lib().seg_attn_workspace_bytes(ctypes.byref(lay.sizes), dt, hq, hkv, d, int(bwd))
    return torch.empty(max(n, 1), dtype=torch.uint8, device=lay.device)


def seg_attn_fwd(lay: Layout, q, k, v, softmax_scale: float, o=None, lse=None, ws=None):
    """Masked GQA attention forward; q [P, hq, d], k/v [P, hkv, d]."""
    import torch
    P, hq, d = q.shape
    hkv = k.shape[1]
    dt = _dtype_code(q)
    assert q.is_contiguous() and k.is_contiguous() and v.is_contiguous()
    assert k.dtype == q.dtype == v.dtype
    if o is None:
        o = torch.empty_like(q)
    if lse is None:
        lse = torch.empty((hq, P), dtype=torch.float32, device=q.device)
    if ws is None:
        ws = attn_workspace(lay, dt, hq, hkv, d, False)
    check(_lib.lib().seg_attn_fwd(ctypes.byref(lay.c), ctypes.byref(lay.sizes), dt, hq, hkv, d,
                                  float(softmax_scale), q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                  o.data_ptr(), lse.data_ptr(), ws.data_ptr(), ws.numel(),
                                  _stream(q.device)))
    return o, lse


def seg_attn_bwd(lay: Layout, q, k, v, o, lse, dout, softmax_scale: float, dq=None, dk=None,
                 dv=None, ws=None):
    """Gradients of sum(O * dout) w.r.t. q, k, v."""
    import torch
    P, hq, d = q.shape
    hkv = k.shape[1]
    dt = _dtype_code(q)
    for t in (q, k, v, o, dout):
        assert t.is_contiguous() and t.dtype == q.dtype
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    if ws is None:
        ws = attn_workspace(lay, dt, hq, hkv, d, True)
    check(_lib.lib().seg_attn_bwd(ctypes.byref(lay.c), ctypes.byref(lay.sizes), dt, hq, hkv, d,
                                  float(softmax_scale), q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                  o.data_ptr(), lse.data_ptr(), dout.data_ptr(), dq.data_ptr(),
                                  dk.data_ptr(), dv.data_ptr(), ws.data_ptr(), ws.numel(),
                                  _stream(q.device)))
    return dq, dk, dv


def seg_attn_bwd_noalloc(lay: Layout, q, k, v, o, lse, dout, softmax_scale: float, dq, dk, dv):
    """seg_attn_bwd on the library's fixed device scratch: the caller passes
    every output, nothing is allocated (calls on one GPU must not overlap)."""
    dt = _dtype_code(q)
    P, hq, d = q.shape
    hkv = k.shape[1]
    for t in (q, k, v, o, dout, dq):
        assert t.is_contiguous() and t.dtype == q.dtype
    for t in (dk, dv):
        assert t.is_contiguous() and t.dtype == q.dtype
    check(_lib.lib().seg_attn_bwd_noalloc(ctypes.byref(lay.c), ctypes.byref(lay.sizes), dt, hq,
                                          hkv, d, float(softmax_scale), q.data_ptr(),
                                          k.data_ptr(), v.data_ptr(), o.data_ptr(),
                                          lse.data_ptr(), dout.data_ptr(), dq.data_ptr(),
                                          dk.data_ptr(), dv.data_ptr(), _stream(q.device)))
    return dq, dk, dv


@dataclasses.dataclass
class LossCfg:
    eps_low: float = 0.2
    eps_high: float = 0.2
    dual_clip_c: float = 0.0
    loss_scale: float = 1.0
    logit_scale: float = 1.0
    want_grad: bool = True
    kl_coef: float = 0.0

    def c(self) -> SegLossCfg:
        return SegLossCfg(self.eps_low, self.eps_high, self.dual_clip_c, self.loss_scale,
                          self.logit_scale, int(self.want_grad), self.kl_coef)


def logprob_workspace(rows, hidden, vocab, dt, device):
    import torch
    n = _lib.lib().seg_logprob_workspace_bytes(rows, hidden, vocab, dt)
    return torch.empty(max(n, 1), dtype=torch.uint8, device=device)


def seg_logprob_loss(h, row_index, w, target, old_logp, adv, row_traj, cfg: LossCfg, out=None,
                     ws=None, ref_logp=None):
    """Fused log-prob + clipped-ratio loss with KL penalty (+ gradients when
    cfg.want_grad).

    h [n_h, H]; row_index [R] int32 device or None; w [V, H]; target [R] int32;
    old_logp [R] fp32; adv [num_traj] fp32; row_traj [R] int32; ref_logp [R]
    fp32 or None (needed when cfg.kl_coef > 0).
    Returns dict(logp, loss_tok, clipped, kl_tok, loss_sum, dh, dw).
    """
    import torch
    dev = h.device
    R = int(target.numel())
    V, H = w.shape
    dt = _dtype_code(h)
    assert w.dtype == h.dtype and h.is_contiguous() and w.is_contiguous()
    if out is None:
        out = {
            "logp": torch.empty(max(R, 1), dtype=torch.float32, device=dev),
            "loss_tok": torch.empty(max(R, 1), dtype=torch.float32, device=dev),
            "clipped": torch.empty(max(R, 1), dtype=torch.uint8, device=dev),
            "kl_tok": torch.empty(max(R, 1), dtype=torch.float32, device=dev),
            "loss_sum": torch.empty(1, dtype=torch.float32, device=dev),
            "dh": torch.empty((max(R, 1), H), dtype=h.dtype, device=dev) if cfg.want_grad else None,
            "dw": torch.empty((V, H), dtype=torch.float32, device=dev) if cfg.want_grad else None,
        }
    if ws is None:
        ws = logprob_workspace(R, H, V, dt, dev)
    check(_lib.lib().seg_logprob_loss(
        R, H, V, dt, h.data_ptr(), _ptr(row_index), w.data_ptr(), target.data_ptr(),
        old_logp.data_ptr(), _ptr(ref_logp), adv.data_ptr(), row_traj.data_ptr(),
        int(adv.numel()), ctypes.byref(cfg.c()), out["logp"].data_ptr(),
        out["loss_tok"].data_ptr(), out["clipped"].data_ptr(), _ptr(out.get("kl_tok")),
        out["loss_sum"].data_ptr(), _ptr(out["dh"]), _ptr(out["dw"]), ws.data_ptr(), ws.numel(),
        _stream(dev)))
    return out


@dataclasses.dataclass
class LayerCfg:
    """Shape and settings of the decoder layer (seg_layer_cfg)."""
    hidden: int
    inter: int
    hq: int
    hkv: int
    d: int
    rms_eps: float = 1e-6
    rope_base: float = 1e6
    chunk_rows: int = 0

    def c(self) -> "_lib.SegLayerCfg":
        return _lib.SegLayerCfg(self.hidden, self.inter, self.hq, self.hkv, self.d, self.rms_eps,
                                self.rope_base, self.chunk_rows)


def layer_workspace(lay: Layout, cfg: LayerCfg, bwd: bool):
    import torch
    n = _lib.lib().seg_layer_workspace_bytes(ctypes.byref(lay.sizes), ctypes.byref(cfg.c()),
                                             int(bwd))
    return torch.empty(max(n, 1), dtype=torch.uint8, device=lay.device)


def _layer_weights(w: dict):
    return _lib.SegLayerWeights(*[w[n].data_ptr() for n in _lib.LAYER_WEIGHTS])


def seg_layer_fwd(lay: Layout, cfg: LayerCfg, w: dict, x, y=None, saved=None, ws=None):
    """Decoder-layer forward over the packed rows; x [P, H] bf16, w: the bf16
    weights by name (g1, wq, wk, wv, wo, g2, wg, wu, wd).  Returns (y, saved)."""
    import torch
    P, H = x.shape
    dev = x.device
    assert x.dtype == torch.bfloat16 and x.is_contiguous()
    for n in _lib.LAYER_WEIGHTS:
        assert w[n].dtype == torch.bfloat16 and w[n].is_contiguous(), n
    if y is None:
        y = torch.empty_like(x)
    if saved is None:
        bf = dict(dtype=torch.bfloat16, device=dev)
        saved = {"q": torch.empty((P, cfg.hq, cfg.d), **bf), "k": torch.empty((P, cfg.hkv, cfg.d), **bf),
                 "v": torch.empty((P, cfg.hkv, cfg.d), **bf), "o": torch.empty((P, cfg.hq, cfg.d), **bf),
                 "lse": torch.empty((cfg.hq, P), dtype=torch.float32, device=dev),
                 "y1": torch.empty((P, H), **bf),
                 "rstd1": torch.empty(P, dtype=torch.float32, device=dev),
                 "rstd2": torch.empty(P, dtype=torch.float32, device=dev)}
    sv = _lib.SegLayerSaved(*[saved[n].data_ptr() for n in ("q", "k", "v", "o", "lse", "y1", "rstd1",
                                                             "rstd2")])
    if ws is None:
        ws = layer_workspace(lay, cfg, False)
    check(_lib.lib().seg_layer_fwd(ctypes.byref(lay.c), ctypes.byref(lay.sizes), ctypes.byref(cfg.c()),
                                   ctypes.byref(_layer_weights(w)), x.data_ptr(), y.data_ptr(),
                                   ctypes.byref(sv), ws.data_ptr(), ws.numel(), _stream(dev)))
    return y, saved


def seg_layer_bwd(lay: Layout, cfg: LayerCfg, w: dict, x, saved: dict, dy, dx=None, grads=None,
                  ws=None):
    """Decoder-layer backward: returns (dx, grads) with fp32 weight gradients by name."""
    import torch
    dev = x.device
    assert dy.dtype == torch.bfloat16 and dy.is_contiguous() and dy.shape == x.shape
    if dx is None:
        dx = torch.empty_like(x)
    if grads is None:
        grads = {n: torch.empty(w[n].shape, dtype=torch.float32, device=dev) for n in _lib.LAYER_WEIGHTS}
    sv = _lib.SegLayerSaved(*[saved[n].data_ptr() for n in ("q", "k", "v", "o", "lse", "y1", "rstd1",
                                                             "rstd2")])
    g = _lib.SegLayerGrads(*[grads[n].data_ptr() for n in _lib.LAYER_WEIGHTS])
    if ws is None:
        ws = layer_workspace(lay, cfg, True)
    check(_lib.lib().seg_layer_bwd(ctypes.byref(lay.c), ctypes.byref(lay.sizes), ctypes.byref(cfg.c()),
                                   ctypes.byref(_layer_weights(w)), x.data_ptr(), ctypes.byref(sv),
                                   dy.data_ptr(), dx.data_ptr(), ctypes.byref(g), ws.data_ptr(),
                                   ws.numel(), _stream(dev)))
    return dx, grads


def _device(*tensors):
    """The GPU that all the tensors (None: left out) are on."""
    dev = tensors[0].device
    assert dev.type == "cuda", f"tensors on {dev}"
    index = dev.index
    for t in tensors:
        assert t is None or t.get_device() == index, f"tensors on {dev} and {t.device}"
    return dev


def _current(dev) -> int:
    """The handle of the GPU's current stream (as _stream, without the 2 us of making a
    Stream object of it)."""
    import torch
    return torch._C._cuda_getCurrentRawStream(dev.index)


def _on(dev):
    """Calls are made with the tensors' GPU as the current one."""
    import torch
    if torch._C._cuda_getDevice() == dev.index:
        return _HERE
    return torch.cuda.device(dev)


_HERE = contextlib.nullcontext()


@dataclasses.dataclass
class MropeCfg:
    """Rotary positions on three axes: pairs that turn with time, height and
    width (they sum to d / 2), and the base."""
    sections: tuple
    base: float = 1e6

    def c(self) -> "_lib.SegMropeCfg":
        if len(self.sections) != 3:
            raise ValueError("sections: three numbers (time, height, width)")
        return _lib.SegMropeCfg((ctypes.c_int32 * 3)(*self.sections), self.base)


def seg_mrope_positions(problem: Problem, lay: Layout, grid, pos=None, ws=None):
    """Time, height and width positions [3, P] int32 (-1 in padding rows) of a
    problem's packed layout; grid: host [num_steps, 4] int32, the frames, patch
    rows, patch columns and time step of each step's screenshot (None where no
    step has one)."""
    import torch
    L = _lib.lib()
    pc = problem.c()
    if grid is not None:
        grid = np.ascontiguousarray(np.asarray(grid, dtype=np.int32))
        if grid.shape != (lay.sizes.num_steps, 4):
            raise ValueError(f"grid of shape {grid.shape}, not ({lay.sizes.num_steps}, 4)")
    if pos is None:
        pos = torch.empty((3, lay.sizes.packed_tokens), dtype=torch.int32, device=lay.device)
    assert pos.dtype == torch.int32 and pos.is_contiguous() and pos.shape == (3, lay.sizes.packed_tokens)
    if ws is None:
        n = L.seg_mrope_positions_workspace_bytes(ctypes.byref(pc), ctypes.byref(lay.sizes))
        ws = torch.empty(max(n, 1), dtype=torch.uint8, device=lay.device)
    dev = _device(pos, ws)
    with _on(dev):
        check(L.seg_mrope_positions(ctypes.byref(pc), ctypes.byref(lay.sizes),
                                    None if grid is None else grid.ctypes.data, pos.data_ptr(),
                                    ws.data_ptr(), ws.numel(), _current(dev)))
    return pos


def _heads(t, rows, d, dtype):
    """Heads of t [rows, heads, d] (side by side in a row) and elements between rows."""
    _, heads, last = t.shape
    step, head, one = t.stride()
    assert t.shape[0] == rows and last == d and t.dtype == dtype
    assert one == 1 and (head == d or heads <= 1), "heads of a row must be adjacent"
    return heads, step if rows > 1 else heads * d


def _mrope(f, q, k, pos, cfg: MropeCfg, q_out, k_out):
    import torch
    rows, _, d = q.shape
    dt, dtype = _dtype_code(q), q.dtype
    hq, ldq = _heads(q, rows, d, dtype)
    hkv, ldk = (0, 0) if k is None else _heads(k, rows, d, dtype)
    if q_out is None:
        q_out, ldqo = q.new_empty((rows, hq, d)), hq * d
    else:
        heads, ldqo = _heads(q_out, rows, d, dtype)
        assert heads == hq
    if k is None:
        k_out, ldko = None, 0
    elif k_out is None:
        k_out, ldko = k.new_empty((rows, hkv, d)), hkv * d
    else:
        heads, ldko = _heads(k_out, rows, d, dtype)
        assert heads == hkv
    assert pos.shape == (3, rows) and pos.dtype == torch.int32 and pos.is_contiguous()
    dev = _device(q, k, q_out, k_out, pos)
    with _on(dev):
        check(f(rows, dt, ctypes.byref(cfg.c()), hq, hkv, d, pos.data_ptr(), q.data_ptr(), ldq,
                _ptr(k), ldk, q_out.data_ptr(), ldqo, _ptr(k_out), ldko, _current(dev)))
    return q_out, k_out


def seg_mrope_fwd(q, k, pos, cfg: MropeCfg, q_out=None, k_out=None):
    """q [rows, hq, d] and k [rows, hkv, d] (or None) rotated by pos [3, rows]
    int32; rows may lie at any distance, outputs may be the inputs.  Returns
    (q_out, k_out)."""
    return _mrope(_lib.lib().seg_mrope_fwd, q, k, pos, cfg, q_out, k_out)


def seg_mrope_bwd(dq, dk, pos, cfg: MropeCfg, dq_out=None, dk_out=None):
    """Gradients of the unrotated q and k from those of the rotated ones."""
    return _mrope(_lib.lib().seg_mrope_bwd, dq, dk, pos, cfg, dq_out, dk_out)


@dataclasses.dataclass
class Act8:
    """Activations in 8 bits: code [rows, cols] int8 and exp [rows, ceil(cols / 32)]
    uint8, value = code * 2^(exp - 127)."""
    code: object
    exp: object

    @classmethod
    def empty(cls, rows: int, cols: int, device) -> "Act8":
        import torch
        return cls(torch.empty((rows, cols), dtype=torch.int8, device=device),
                   torch.empty((rows, -(-cols // 32)), dtype=torch.uint8, device=device))

    def c(self) -> "_lib.SegAct8":
        import torch
        rows, cols = self.code.shape
        assert self.code.dtype == torch.int8 and self.exp.dtype == torch.uint8
        assert self.exp.shape == (rows, -(-cols // 32))
        assert self.code.is_contiguous() and self.exp.is_contiguous()
        return _lib.SegAct8(self.code.data_ptr(), self.exp.data_ptr())


def _rows(t) -> int:
    """Elements between the rows of t [rows, cols]."""
    rows, cols = t.shape
    assert cols <= 1 or t.stride(1) == 1, "columns must be adjacent"
    return cols if rows <= 1 else t.stride(0)


def seg_act_pack(x, out: Optional[Act8] = None) -> Act8:
    """x [rows, cols] (rows at any distance) in 8 bits."""
    rows, cols = x.shape
    dt = _dtype_code(x)
    if out is None:
        import torch
        out = Act8(x.new_empty((rows, cols), dtype=torch.int8),
                   x.new_empty((rows, -(-cols // 32)), dtype=torch.uint8))
    assert out.code.shape == (rows, cols)
    dev = _device(x, out.code, out.exp)
    with _on(dev):
        check(_lib.lib().seg_act_pack(rows, cols, dt, x.data_ptr(), _rows(x), ctypes.byref(out.c()),
                                      _current(dev)))
    return out


def seg_act_unpack(act: Act8, dtype=None, x=None):
    """The values of `act` in `dtype` (bf16 by default), or into x [rows, cols]."""
    import torch
    rows, cols = act.code.shape
    if x is None:
        x = torch.empty((rows, cols), dtype=dtype or torch.bfloat16, device=act.code.device)
    assert x.shape == (rows, cols) and (dtype is None or x.dtype == dtype)
    dev = _device(x, act.code, act.exp)
    with _on(dev):
        check(_lib.lib().seg_act_unpack(rows, cols, _dtype_code(x), ctypes.byref(act.c()),
                                        x.data_ptr(), _rows(x), _current(dev)))
    return x


def _glu_args(x, wg, wu):
    import torch
    rows, hidden = x.shape
    inter = wg.shape[0]
    for t in (wg, wu):
        assert t.shape == (inter, hidden) and t.dtype == torch.bfloat16 and t.is_contiguous()
    assert x.dtype == torch.bfloat16
    return rows, hidden, inter


def _kept(kept, rows, inter):
    """The two C structs of a kept pair, and its tensors."""
    if kept is None:
        return (None, None), ()
    g, u = kept
    assert g.code.shape == u.code.shape == (rows, inter)
    return (ctypes.byref(g.c()), ctypes.byref(u.c())), (g.code, g.exp, u.code, u.exp)


def glu_workspace(rows, hidden, inter, bwd: bool, kept: bool, device):
    import torch
    n = _lib.lib().seg_glu_workspace_bytes(rows, hidden, inter, int(bwd), int(kept))
    return torch.empty(max(n, 1), dtype=torch.uint8, device=device)


def seg_glu_fwd(x, wg, wu, keep=False, m=None, ws=None):
    """m = silu(x wg^T) * (x wu^T); x [rows, H] (rows at any distance), wg and wu
    [I, H], bf16.  keep: True, or a pair (Act8, Act8) to fill, keeps the gate and
    up values in 8 bits.  Returns (m, kept or None)."""
    import torch
    rows, hidden, inter = _glu_args(x, wg, wu)
    if m is None:
        m = x.new_empty((rows, inter))
    assert m.shape == (rows, inter) and m.dtype == torch.bfloat16 and m.is_contiguous()
    if keep is True:
        keep = (Act8.empty(rows, inter, x.device), Act8.empty(rows, inter, x.device))
    kept = keep or None
    c, tensors = _kept(kept, rows, inter)
    if ws is None:
        ws = glu_workspace(rows, hidden, inter, False, False, x.device)
    dev = _device(x, wg, wu, m, ws, *tensors)
    with _on(dev):
        check(_lib.lib().seg_glu_fwd(rows, hidden, inter, x.data_ptr(), _rows(x), wg.data_ptr(),
                                     wu.data_ptr(), m.data_ptr(), *c, ws.data_ptr(), ws.numel(),
                                     _current(dev)))
    return m, kept


def seg_glu_bwd(x, wg, wu, dm, kept=None, dw_dtype=None, want_m=True, out=None, ws=None):
    """Gradients of sum(m * dm); kept: seg_glu_fwd's pair, or None to compute the
    gate and up values again.  Returns dict(dx, dwg, dwu, m): the weight gradients
    in dw_dtype (fp32 by default), m again unless want_m is false (then None)."""
    import torch
    rows, hidden, inter = _glu_args(x, wg, wu)
    assert dm.shape == (rows, inter) and dm.dtype == torch.bfloat16 and dm.is_contiguous()
    dev = x.device
    if out is None:
        dw = dict(dtype=dw_dtype or torch.float32, device=dev)
        bf = dict(dtype=torch.bfloat16, device=dev)
        out = {"dx": torch.empty((rows, hidden), **bf), "dwg": torch.empty((inter, hidden), **dw),
               "dwu": torch.empty((inter, hidden), **dw),
               "m": torch.empty((rows, inter), **bf) if want_m else None}
    assert out["dwg"].dtype == out["dwu"].dtype
    for n, shape in (("dx", (rows, hidden)), ("dwg", (inter, hidden)), ("dwu", (inter, hidden)),
                     ("m", (rows, inter))):
        t = out.get(n)
        assert (n == "m" and t is None) or (t.shape == shape and t.is_contiguous()), n
        assert t is None or n in ("dwg", "dwu") or t.dtype == torch.bfloat16, n
    if ws is None:
        ws = glu_workspace(rows, hidden, inter, True, kept is not None, dev)
    c, tensors = _kept(kept, rows, inter)
    _device(x, wg, wu, dm, out["dx"], out["dwg"], out["dwu"], out.get("m"), ws, *tensors)
    with _on(dev):
        check(_lib.lib().seg_glu_bwd(rows, hidden, inter, x.data_ptr(), _rows(x), wg.data_ptr(),
                                     wu.data_ptr(), *c, dm.data_ptr(), _ptr(out.get("m")),
                                     out["dx"].data_ptr(), _dtype_code(out["dwg"]),
                                     out["dwg"].data_ptr(), out["dwu"].data_ptr(), ws.data_ptr(),
                                     ws.numel(), _current(dev)))
    return out


def _saved8_widths(cfg: LayerCfg) -> dict:
    return {"x": cfg.hidden, "y1": cfg.hidden, "q": cfg.hq * cfg.d, "o": cfg.hq * cfg.d,
            "k": cfg.hkv * cfg.d, "v": cfg.hkv * cfg.d, "g": cfg.inter, "u": cfg.inter}


def layer_saved8(lay: Layout, cfg: LayerCfg, keep_gate=False) -> dict:
    """Empty 8-bit saved activations of the layer over `lay` (Act8 by name, and the
    fp32 vectors lse, rstd1 and rstd2); keep_gate: with the gate and up values."""
    import torch
    P, dev = lay.sizes.packed_tokens, lay.device
    out = {n: Act8.empty(P, c, dev) for n, c in _saved8_widths(cfg).items()
           if keep_gate or n not in ("g", "u")}
    out.update(lse=torch.empty((cfg.hq, P), dtype=torch.float32, device=dev),
               rstd1=torch.empty(P, dtype=torch.float32, device=dev),
               rstd2=torch.empty(P, dtype=torch.float32, device=dev))
    return out


def _layer_ext(lay, cfg, rope, pos, saved8):
    """The C struct, and the tensors that have to be on the layer's GPU with it."""
    import torch
    P = lay.sizes.packed_tokens
    e, tensors = _lib.SegLayerExt(), [lay.tok_meta]
    assert rope is not None or pos is None, "pos needs rope"
    if rope is not None:
        assert pos is not None, "rope needs pos"
        assert pos.shape == (3, P) and pos.dtype == torch.int32 and pos.is_contiguous()
        e.rope = ctypes.pointer(rope.c())
        e.pos = pos.data_ptr()
        tensors.append(pos)
    if saved8 is not None:
        want = _saved8_widths(cfg)
        s = _lib.SegLayerSaved8()
        for n in _lib.SAVED8:
            a = saved8.get(n)
            if a is None:
                assert n in ("g", "u"), f"saved8 has no {n}"
                continue
            assert a.code.shape == (P, want[n]), n
            setattr(s, n, a.c())
            tensors += [a.code, a.exp]
        for n, size in (("lse", cfg.hq * P), ("rstd1", P), ("rstd2", P)):
            t = saved8[n]
            assert t.numel() == size and t.is_contiguous() and t.dtype == torch.float32, n
            setattr(s, n, t.data_ptr())
            tensors.append(t)
        e.saved8 = ctypes.pointer(s)
    return e, tensors


def layer_ext_workspace(lay: Layout, cfg: LayerCfg, saved8: bool, bwd: bool):
    import torch
    n = _lib.lib().seg_layer_ext_workspace_bytes(ctypes.byref(lay.sizes), ctypes.byref(cfg.c()),
                                                 int(saved8), int(bwd))
    return torch.empty(max(n, 1), dtype=torch.uint8, device=lay.device)


def _layer_saved(saved, cfg, P, H, dev):
    """The bf16 saved buffers (allocated where None) and their C struct."""
    import torch
    shapes = {"q": (P, cfg.hq, cfg.d), "k": (P, cfg.hkv, cfg.d), "v": (P, cfg.hkv, cfg.d),
              "o": (P, cfg.hq, cfg.d), "lse": (cfg.hq, P), "y1": (P, H), "rstd1": (P,), "rstd2": (P,)}
    f32 = ("lse", "rstd1", "rstd2")
    if saved is None:
        saved = {n: torch.empty(s, dtype=torch.float32 if n in f32 else torch.bfloat16, device=dev)
                 for n, s in shapes.items()}
    for n, s in shapes.items():
        assert saved[n].shape == s and saved[n].is_contiguous(), n
        assert saved[n].dtype == (torch.float32 if n in f32 else torch.bfloat16), n
    return saved, _lib.SegLayerSaved(*[saved[n].data_ptr() for n in shapes])


def _layer_args(lay, cfg, w, x):
    import torch
    assert x.shape == (lay.sizes.packed_tokens, cfg.hidden)
    assert x.dtype == torch.bfloat16 and x.is_contiguous()
    H, I, QD, KD = cfg.hidden, cfg.inter, cfg.hq * cfg.d, cfg.hkv * cfg.d
    shapes = {"g1": (H,), "wq": (QD, H), "wk": (KD, H), "wv": (KD, H), "wo": (H, QD), "g2": (H,),
              "wg": (I, H), "wu": (I, H), "wd": (H, I)}
    for n in _lib.LAYER_WEIGHTS:
        assert w[n].shape == shapes[n] and w[n].dtype == torch.bfloat16 and w[n].is_contiguous(), n
    return [w[n] for n in _lib.LAYER_WEIGHTS]


def seg_layer_fwd_ext(lay: Layout, cfg: LayerCfg, w: dict, x, rope: Optional[MropeCfg] = None,
                      pos=None, saved8=None, y=None, saved=None, ws=None):
    """seg_layer_fwd with positions on three axes (rope, pos [3, P] int32) and 8-bit
    saved activations (saved8: layer_saved8's dict, filled here; y may then be x).
    Returns (y, saved8), or (y, saved) without saved8."""
    import torch
    P, H = x.shape
    weights = _layer_args(lay, cfg, w, x)
    e, tensors = _layer_ext(lay, cfg, rope, pos, saved8)
    if y is None:
        y = torch.empty_like(x)
    assert y.shape == x.shape and y.dtype == x.dtype and y.is_contiguous()
    sv = None
    if saved8 is None:
        saved, c = _layer_saved(saved, cfg, P, H, x.device)
        sv = ctypes.byref(c)
        tensors += list(saved.values())
    if ws is None:
        ws = layer_ext_workspace(lay, cfg, saved8 is not None, False)
    dev = _device(x, y, ws, *weights, *tensors)
    with _on(dev):
        check(_lib.lib().seg_layer_fwd_ext(
            ctypes.byref(lay.c), ctypes.byref(lay.sizes), ctypes.byref(cfg.c()), ctypes.byref(e),
            ctypes.byref(_layer_weights(w)), x.data_ptr(), y.data_ptr(), sv, ws.data_ptr(),
            ws.numel(), _current(dev)))
    return y, saved if saved8 is None else saved8


def seg_layer_bwd_ext(lay: Layout, cfg: LayerCfg, w: dict, dy, rope: Optional[MropeCfg] = None,
                      pos=None, saved8=None, x=None, saved=None, dx=None, grads=None, ws=None):
    """seg_layer_bwd with rope and pos of the forward, from saved8 alone (dx may then be
    dy) or from x and saved: returns (dx, grads) with fp32 weight gradients by name."""
    import torch
    weights = _layer_args(lay, cfg, w, dy)
    dev, (P, H) = dy.device, dy.shape
    e, tensors = _layer_ext(lay, cfg, rope, pos, saved8)
    sv = None
    if saved8 is None:
        assert x is not None and saved is not None, "the backward needs saved8, or x and saved"
        assert x.shape == dy.shape and x.dtype == dy.dtype and x.is_contiguous()
        saved, c = _layer_saved(saved, cfg, P, H, dev)
        sv = ctypes.byref(c)
        tensors += [x, *saved.values()]
    if dx is None:
        dx = torch.empty_like(dy)
    assert dx.shape == dy.shape and dx.dtype == dy.dtype and dx.is_contiguous()
    if grads is None:
        grads = {n: torch.empty(w[n].shape, dtype=torch.float32, device=dev) for n in _lib.LAYER_WEIGHTS}
    for n in _lib.LAYER_WEIGHTS:
        assert grads[n].shape == w[n].shape and grads[n].dtype == torch.float32, n
        assert grads[n].is_contiguous(), n
    if ws is None:
        ws = layer_ext_workspace(lay, cfg, saved8 is not None, True)
    _device(dy, dx, ws, *weights, *tensors, *grads.values())
    g = _lib.SegLayerGrads(*[grads[n].data_ptr() for n in _lib.LAYER_WEIGHTS])
    with _on(dev):
        check(_lib.lib().seg_layer_bwd_ext(
            ctypes.byref(lay.c), ctypes.byref(lay.sizes), ctypes.byref(cfg.c()), ctypes.byref(e),
            ctypes.byref(_layer_weights(w)), None if saved8 is not None else x.data_ptr(), sv,
            dy.data_ptr(), dx.data_ptr(), ctypes.byref(g), ws.data_ptr(), ws.numel(), _current(dev)))
    return dx, grads


def _up(n: int, to: int) -> int:
    return -(-n // to) * to


@dataclasses.dataclass
class Fp8:
    """A tensor [rows, cols] in 8-bit floating point (e4m3) with a power of two for each
    block of block_rows (1 or 128) rows x 128 columns: code [rows, cols up to 16] uint8
    (zero codes behind cols) and exp [ceil(cols / 128), ceil(rows / block_rows) up to 16]
    uint8, value = number(code) * 2^(exp - 127)."""
    code: object
    exp: object
    cols: int
    block_rows: int = 1

    @classmethod
    def empty(cls, rows: int, cols: int, block_rows: int, device) -> "Fp8":
        import torch
        if block_rows not in (1, 128):
            raise ValueError(f"blocks of {block_rows} rows, not of 1 or 128")
        return cls(torch.empty((rows, _up(cols, 16)), dtype=torch.uint8, device=device),
                   torch.empty((-(-cols // 128), _up(-(-rows // block_rows), 16)), dtype=torch.uint8, device=device),
                   cols, block_rows)

    @property
    def shape(self):
        return self.code.shape[0], self.cols

    def c(self) -> "_lib.SegFp8":
        import torch
        code, exp, cols, br, u8 = self.code, self.exp, self.cols, self.block_rows, torch.uint8
        rows = code.shape[0]
        assert br in (1, 128)
        assert code.dtype == u8 and exp.dtype == u8
        assert code.shape == (rows, _up(cols, 16))
        assert exp.shape == (-(-cols // 128), _up(-(-rows // br), 16))
        assert code.is_contiguous() and exp.is_contiguous()
        return _lib.SegFp8(code.data_ptr(), exp.data_ptr(), br)


def seg_fp8_pack(x, block_rows: int = 1, out: Optional[Fp8] = None) -> Fp8:
    """x [rows, cols] (rows at any distance) in 8-bit floating point: a scale for each
    128 columns of a row, or (block_rows = 128) of 128 rows, as weights have them."""
    import torch
    rows, cols = x.shape
    dt = _dtype_code(x)
    if out is None:
        if block_rows not in (1, 128):
            raise ValueError(f"blocks of {block_rows} rows, not of 1 or 128")
        u8 = torch.uint8
        out = Fp8(x.new_empty((rows, _up(cols, 16)), dtype=u8),
                  x.new_empty((-(-cols // 128), _up(-(-rows // block_rows), 16)), dtype=u8), cols, block_rows)
        c = _lib.SegFp8(out.code.data_ptr(), out.exp.data_ptr(), block_rows)
    else:
        assert out.shape == (rows, cols) and out.block_rows == block_rows
        c = out.c()
    dev = _device(x, out.code, out.exp)
    with _on(dev):
        check(_lib.lib().seg_fp8_pack(rows, cols, dt, x.data_ptr(), _rows(x), ctypes.byref(c), _current(dev)))
    return out


def seg_fp8_unpack(a: Fp8, dtype=None, x=None):
    """The values of `a` in `dtype` (bf16 by default), or into x [rows, cols]."""
    import torch
    rows, cols = a.shape
    if x is None:
        x = a.code.new_empty((rows, cols), dtype=dtype or torch.bfloat16)
    assert x.shape == (rows, cols) and (dtype is None or x.dtype == dtype)
    dev = _device(x, a.code, a.exp)
    with _on(dev):
        check(_lib.lib().seg_fp8_unpack(rows, cols, _dtype_code(x), ctypes.byref(a.c()), x.data_ptr(), _rows(x),
                                        _current(dev)))
    return x


def fp8_gemm_workspace(rows: int, outs: int, cols: int, device):
    import torch
    n = _lib.lib().seg_fp8_gemm_workspace_bytes(rows, outs, cols)
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def seg_fp8_gemm(a: Fp8, b: Fp8, dtype=None, y=None, ws=None):
    """y [rows, outs] = a b^T of a [rows, cols] and b [outs, cols] in 8-bit floating point,
    in `dtype` (bf16 by default), or into y (rows at any distance)."""
    import torch
    rows, cols = a.shape
    outs = b.shape[0]
    assert b.shape == (outs, cols), f"a has {cols} columns and b {b.shape[1]}"
    if y is None:
        y = a.code.new_empty((rows, outs), dtype=dtype or torch.bfloat16)
    assert y.shape == (rows, outs) and (dtype is None or y.dtype == dtype)
    if ws is None:
        ws = fp8_gemm_workspace(rows, outs, cols, y.device)
    dev = _device(y, a.code, a.exp, b.code, b.exp, ws)
    with _on(dev):
        check(_lib.lib().seg_fp8_gemm(rows, outs, cols, ctypes.byref(a.c()), ctypes.byref(b.c()), _dtype_code(y),
                                      y.data_ptr(), _rows(y), _ptr(ws), 0 if ws is None else ws.numel(),
                                      _current(dev)))
    return y


def top_logits_workspace(rows: int, vocab: int, device):
    import torch
    n = _lib.lib().seg_top_logits_workspace_bytes(rows, vocab)
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def seg_top_logits(z, k: int, scale: float = 1.0, out: Optional[dict] = None, ws=None) -> dict:
    """The k largest of each row of z [rows, vocab] (rows at any distance): dict(ids
    [rows, k] int32, logits [rows, k] fp32, both by value and then column; lse [rows]
    fp32, the log-sum-exp of scale * z over the whole row)."""
    import torch
    rows, vocab = z.shape
    dt, dev = _dtype_code(z), z.device
    if out is None:
        out = {"ids": z.new_empty((rows, k), dtype=torch.int32), "logits": z.new_empty((rows, k), dtype=torch.float32),
               "lse": z.new_empty(rows, dtype=torch.float32)}
    else:
        for n, shape, dtype in (("ids", (rows, k), torch.int32), ("logits", (rows, k), torch.float32),
                                ("lse", (rows,), torch.float32)):
            assert out[n].shape == shape and out[n].dtype == dtype and out[n].is_contiguous(), n
    if ws is None:
        ws = top_logits_workspace(rows, vocab, dev)
    _device(z, out["ids"], out["logits"], out["lse"], ws)
    with _on(dev):
        check(_lib.lib().seg_top_logits(rows, vocab, k, dt, z.data_ptr(), _rows(z), scale, out["ids"].data_ptr(),
                                        out["logits"].data_ptr(), out["lse"].data_ptr(), _ptr(ws),
                                        0 if ws is None else ws.numel(), _current(dev)))
    return out


@dataclasses.dataclass
class DistillCfg:
    """Settings of the distillation loss (seg_distill_cfg)."""
    logit_scale: float = 1.0
    teacher_scale: float = 1.0
    loss_scale: float = 1.0
    want_grad: bool = True

    def c(self) -> "_lib.SegDistillCfg":
        return _lib.SegDistillCfg(self.logit_scale, self.teacher_scale, self.loss_scale, int(self.want_grad))


def distill_workspace(rows: int, hidden: int, vocab: int, k: int, dt: int, want_grad: bool, device):
    import torch
    n = _lib.lib().seg_distill_workspace_bytes(rows, hidden, vocab, k, dt, int(want_grad))
    return torch.empty(max(n, 1), dtype=torch.uint8, device=device)


def seg_distill_loss(h, row_index, w, ids, logits, cfg: DistillCfg, t_lse=None, row_weight=None,
                     dw_dtype=None, out: Optional[dict] = None, ws=None) -> dict:
    """Divergence of the student's distribution from a teacher's top logits, with
    gradients when cfg.want_grad.

    h [n_h, H]; row_index [R] int32 or None; w [V, H]; ids [R, k] int32 (negative: no
    entry) and logits [R, k] fp32, as seg_top_logits returns them; t_lse [R] fp32 or None
    (the teacher's probabilities are then normalised over the entries); row_weight [R]
    fp32 or None.  Returns dict(loss_tok, lse, loss_sum, dh, dw): dw in dw_dtype (fp32 by
    default), dh and dw None without want_grad.
    """
    import torch
    dev = h.device
    (n_h, H), (R, k), V = h.shape, ids.shape, w.shape[0]
    dt = _dtype_code(h)
    assert w.shape == (V, H) and w.dtype == h.dtype and h.is_contiguous() and w.is_contiguous()
    assert ids.dtype == torch.int32 and ids.is_contiguous()
    assert row_index is None or (row_index.shape == (R,) and row_index.dtype == torch.int32 and row_index.is_contiguous())
    assert logits.shape == (R, k) and logits.dtype == torch.float32 and logits.is_contiguous()
    for t in (t_lse, row_weight):
        assert t is None or (t.shape == (R,) and t.dtype == torch.float32 and t.is_contiguous())
    fresh = out is None
    if fresh:
        f32 = torch.float32
        out = {"loss_tok": h.new_empty(R, dtype=f32), "lse": h.new_empty(R, dtype=f32), "loss_sum": h.new_empty(1, dtype=f32),
               "dh": h.new_empty((R, H)) if cfg.want_grad else None,
               "dw": h.new_empty((V, H), dtype=dw_dtype or f32) if cfg.want_grad else None}
    else:
        for n, shape in (("loss_tok", (R,)), ("lse", (R,)), ("loss_sum", (1,))):
            assert out[n].shape == shape and out[n].dtype == torch.float32 and out[n].is_contiguous(), n
    dh, dw = out.get("dh"), out.get("dw")
    if cfg.want_grad and not fresh:
        assert dh.shape == (R, H) and dh.dtype == h.dtype and dh.is_contiguous()
        assert dw.shape == (V, H) and dw.is_contiguous() and (dw_dtype is None or dw.dtype == dw_dtype)
    if ws is None:
        ws = distill_workspace(R, H, V, k, dt, cfg.want_grad, dev)
    _device(h, w, ids, logits, row_index, t_lse, row_weight, dh, dw, ws, *(out[n] for n in ("loss_tok", "lse", "loss_sum")))
    with _on(dev):
        check(_lib.lib().seg_distill_loss(
            R, H, V, k, dt, n_h, h.data_ptr(), _ptr(row_index), w.data_ptr(), ids.data_ptr(), logits.data_ptr(),
            _ptr(t_lse), _ptr(row_weight), ctypes.byref(cfg.c()), out["loss_tok"].data_ptr(), out["lse"].data_ptr(),
            out["loss_sum"].data_ptr(), _ptr(dh), _dtype_code(dw) if cfg.want_grad else 0, _ptr(dw), ws.data_ptr(),
            ws.numel(), _current(dev)))
    return out
