"""Distillation from a teacher's top logits on the GPU against the float64 oracle.

Forward: h and w are bf16 (fp32 ones are rounded to it first, here too), products exact,
a logit's fp32 sum is off by at most e_z = (H + 2) 2^-24 s sum|h w|; the log-sum-exp by the
largest e_z and (log V + |lse| + 20) 2^-22 for its exponentials and sums; t = scale
logits, its norm and their difference by (|t| + |norm| + 4) 2^-22; a term p (log p - z +
lse) by p times these and p's own (|log p| + 4) 2^-22 of itself.

Backward: dz rounds to bf16 (2^-8 of itself, and what e_z, and lse's and norm's errors, move
it), its products with w and h are exact, their sums in fp32, and the results round again
where they are bf16.  Over a whole tensor the two roundings are independent and uniform,
2^-8 / sqrt(3) each, so the relative Frobenius error stays below 2^-8."""
import numpy as np
import pytest

from oracle import distill as OD
from paper_2607_11185_amd import seg as S
from tests.gpu_helpers import rel, say

pytestmark = pytest.mark.gpu


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def _dt(name):
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def _inputs(rows, hidden, vocab, k, dtype="bf16", seed=0, given=False, spread=1.0):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed * 1000 + rows + vocab)
    h = torch.randn(rows, hidden, generator=gen, device="cuda").to(_dt(dtype))
    w = (torch.randn(vocab, hidden, generator=gen, device="cuda") * (2 * spread / hidden ** 0.5)).to(_dt(dtype))
    ids = torch.argsort(torch.rand(rows, vocab, generator=gen, device="cuda"), dim=1)[:, :k].int().contiguous()
    logits = torch.randn(rows, k, generator=gen, device="cuda") * 2.5 + 3
    t_lse = torch.logsumexp(logits * 0.8, 1) + 0.3 if given else None
    weight = torch.rand(rows, generator=gen, device="cuda") + 0.5
    return h, w, ids, logits, t_lse, weight


def _bf(t):
    """The values that the kernels compute with."""
    import torch
    return t.to(torch.bfloat16).double().cpu().numpy()


LS, TS = 0.9, 0.8


def _oracle(h, w, ids, logits, t_lse, weight, row_index=None, loss_scale=1.0):
    hb = _bf(h)
    if row_index is not None:
        hb = hb[row_index.cpu().numpy()]
    return hb, OD.loss_and_grads(hb, _bf(w), ids.cpu().numpy(), _np(logits), np.float64(np.float32(LS)),
                                 np.float64(np.float32(TS)), loss_scale, _np(t_lse), _np(weight))


def _check(h, w, ids, logits, t_lse, weight, row_index=None, dw="bf16", loss_scale=0.25):
    import torch
    cfg = S.DistillCfg(LS, TS, loss_scale, True)
    out = S.seg_distill_loss(h, row_index, w, ids, logits, cfg, t_lse, weight, dw_dtype=_dt(dw))
    hb, ref = _oracle(h, w, ids, logits, t_lse, weight, row_index, loss_scale)
    wb = _bf(w)
    H, V = w.shape[1], w.shape[0]
    ez = ((H + 2) * 2.0 ** -24 * LS * (np.abs(hb) @ np.abs(wb).T)).max(1)
    el = ez + (np.log(V) + np.abs(ref["lse"]) + 20) * 2.0 ** -22
    err = np.abs(_np(out["lse"]) - ref["lse"])
    assert bool((err <= el).all()), ("lse", float((err / el).max()))
    t = np.where(ids.cpu().numpy() >= 0, _np(logits) * TS, 0)
    t = np.where(np.isfinite(t), t, 0)
    p, logp = OD.teacher(ids.cpu().numpy(), _np(logits), TS, _np(t_lse))
    en = (2 * np.abs(t).max(1) + 12 + (0 if t_lse is None else np.abs(_np(t_lse)))) * 2.0 ** -22
    w_r = np.abs(_np(weight)) if weight is not None else np.ones(len(el))
    size = np.where(p > 0, p * (np.abs(np.where(p > 0, logp, 0)) + np.abs(np.take_along_axis(ref["z"], np.maximum(ids.cpu().numpy(), 0), 1))
                                + np.abs(ref["lse"])[:, None] + 1), 0).sum(1)
    tol = w_r * (p.sum(1) * (ez + el + en) + size * (en + ids.shape[1] * 2.0 ** -24 + 2.0 ** -20)) + 1e-30
    err = np.abs(_np(out["loss_tok"]) - ref["loss_tok"])
    assert bool((err <= tol).all()), ("loss_tok", float((err / tol).max()))
    total = loss_scale * tol.sum() + 2.0 ** -23 * abs(ref["loss_sum"])
    assert abs(float(out["loss_sum"]) - ref["loss_sum"]) <= total
    # no forward of its own: without gradients the same bits
    only = S.seg_distill_loss(h, row_index, w, ids, logits, S.DistillCfg(LS, TS, loss_scale, False), t_lse, weight)
    assert only["dh"] is None and only["dw"] is None
    for n in ("loss_tok", "lse", "loss_sum"):
        assert torch.equal(only[n], out[n]), n
    for n in ("dh", "dw"):
        e = rel(_np(out[n]), ref[n])
        say(n, e)
        assert e < 2.0 ** -8, n
    return out, ref


SHAPES = [(1, 8, 1, 1), (1, 64, 5, 5), (3, 72, 130, 7), (16, 128, 128, 64), (17, 200, 1001, 5), (40, 256, 999, 200), (70, 328, 3000, 256),
          (130, 520, 5003, 33), (300, 128, 300, 1), (33, 1024, 20000, 64)]


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_loss_and_gradients(shape, given):
    say(shape, given)
    _check(*_inputs(*shape, given=given))


@pytest.mark.parametrize("shape", [(3, 72, 130, 7), (40, 256, 999, 200)], ids=lambda s: "x".join(map(str, s)))
def test_fp32_inputs_and_gradients(shape):
    _check(*_inputs(*shape, dtype="f32"), dw="f32")


def test_without_weights_and_large_logits():
    h, w, ids, logits, t_lse, _ = _inputs(40, 128, 700, 12, spread=8.0)
    _check(h, w, ids, logits * 6, t_lse, None)


def test_some_rows_of_a_batch():
    import torch
    h, w, ids, logits, t_lse, weight = _inputs(50, 128, 900, 9)
    more = torch.randn(80, 128, device="cuda").bfloat16()
    index = torch.randperm(80, device="cuda")[:50].int()
    index[7] = index[8]                                   # a row may be used twice
    _check(more, w, ids, logits, t_lse, weight, index)


@pytest.mark.parametrize("given", [False, True])
def test_entries_that_are_not_there(given):
    """Missing, repeated and impossible entries; rows of none."""
    import torch
    h, w, ids, logits, t_lse, weight = _inputs(20, 128, 300, 10, given=given)
    ids[0, 4:] = -1
    ids[1, ::2] = -7
    ids[2] = ids[2, 0]
    ids[3, 5], ids[3, 9] = ids[3, 0], ids[3, 0]
    logits[4, 3:] = -float("inf")
    logits[5, 0] = -float("inf")
    ids[6], logits[7] = -1, -float("inf")
    weight[8] = 0
    logits[9] = -3.0e38
    logits[10, 2:] = torch.finfo(torch.float32).min
    if t_lse is not None:
        t_lse[9] = 0
    out, ref = _check(h, w, ids, logits, t_lse, weight)
    for r in (6, 7, 8):
        assert float(out["loss_tok"][r]) == 0 and not bool(out["dh"][r].any())


def test_rows_that_do_not_count_may_hold_anything():
    """Without weight or entries, NaN and infinities in h, logits, ids and t_lse reach nothing."""
    import torch
    h, w, ids, logits, _, weight = _inputs(40, 128, 300, 10, given=True)
    t_lse = torch.logsumexp(logits * TS, 1)
    keep = torch.ones(40, dtype=torch.bool, device="cuda")
    keep[[3, 17, 39]] = False
    cfg = S.DistillCfg(LS, TS, 1.0, True)
    weight[~keep] = 0
    clean = S.seg_distill_loss(h, None, w, ids, logits, cfg, t_lse, weight)
    h[3], h[17, 5], h[39] = float("nan"), float("inf"), float("nan")
    logits[3], ids[17, 2], ids[17, 3], t_lse[39] = float("nan"), 300, 2 ** 31 - 1, float("nan")
    got = S.seg_distill_loss(h, None, w, ids, logits, cfg, t_lse, weight)
    for n in ("loss_tok", "loss_sum", "dh", "dw"):
        assert torch.equal(got[n], clean[n]), n
    assert torch.equal(got["lse"][keep], clean["lse"][keep])
    ids[17], weight[17] = -1, 1.0                         # no entries, with weight
    got = S.seg_distill_loss(h, None, w, ids, logits, cfg, t_lse, weight)
    for n in ("loss_tok", "dh", "dw"):
        assert torch.equal(got[n], clean[n]), n


def test_bad_rows_are_nan_and_alone():
    """An id past the vocabulary, a row index outside h, a NaN logit: that row's loss and dh."""
    import torch
    h, w, ids, logits, t_lse, weight = _inputs(40, 128, 300, 10)
    index = torch.arange(40, device="cuda", dtype=torch.int32)
    ids[3, 2], index[5], index[6], logits[7, 1] = 300, 40, -1, float("nan")
    out = S.seg_distill_loss(h, index, w, ids, logits, S.DistillCfg(LS, TS), t_lse, weight)
    bad = torch.zeros(40, dtype=torch.bool, device="cuda")
    bad[[3, 5, 6, 7]] = True
    assert torch.equal(out["loss_tok"].isnan(), bad)
    assert torch.equal(out["dh"].isnan().any(1), bad)
    assert bool(out["loss_sum"].isnan())


def test_gradients_against_differences():
    """Of the kernel's own loss along random directions; h moves by whole steps of bf16."""
    import torch
    h, w, ids, logits, _, weight = _inputs(64, 128, 500, 16)
    cfg = S.DistillCfg(LS, TS, 1.0, True)
    out = S.seg_distill_loss(h, None, w, ids, logits, cfg, None, weight)
    gen = torch.Generator(device="cuda").manual_seed(9)
    for name, x in (("dh", h), ("dw", w)):
        step = torch.randn(x.shape, generator=gen, device="cuda") * 0.05 * x.float().abs().mean()
        step += 0.05 * x.float().abs().mean() * out[name].float() / out[name].float().abs().mean()   # not across the slope
        up, down = (x.float() + step).bfloat16(), (x.float() - step).bfloat16()
        loss = []
        for y in (up, down):
            a, b = (y, w) if name == "dh" else (h, y)
            loss.append(S.seg_distill_loss(a, None, b, ids, logits, S.DistillCfg(LS, TS, 1.0, False), None, weight)["loss_sum"])
        want = float((out[name].double() * (up.double() - down.double())).sum())
        got = float(loss[0].double() - loss[1].double())
        say(name, got, want)
        # the third derivative's part (steps of 5 to 10 % of the values) and the roundings
        assert abs(got - want) < 0.03 * abs(want)


def test_large_tensors_past_32_bits():
    """zT past 2^31 bytes and 2^31 elements: rows at both ends against the oracle's softmax."""
    import torch
    rows, hidden, vocab, k = 15000, 64, 150001, 3
    gen = torch.Generator(device="cuda").manual_seed(2)
    h = torch.randn(rows, hidden, generator=gen, device="cuda").bfloat16()
    w = (torch.randn(vocab, hidden, generator=gen, device="cuda") * 0.25).bfloat16()
    ids = torch.randint(0, vocab, (rows, k), generator=gen, device="cuda").int()
    ids[:, 2] = vocab - 1
    logits = torch.randn(rows, k, generator=gen, device="cuda")
    weight = torch.zeros(rows, device="cuda")
    at = torch.tensor([0, 7000, rows - 1], device="cuda")
    weight[at] = 1
    out = S.seg_distill_loss(h, None, w, ids, logits, S.DistillCfg(1.0, 1.0), None, weight, dw_dtype=torch.bfloat16)
    ref = OD.loss_and_grads(_bf(h[at]), _bf(w), ids[at].cpu().numpy(), _np(logits[at]))
    assert rel(_np(out["loss_tok"][at]), ref["loss_tok"]) < 2.0 ** -18
    assert rel(_np(out["dh"][at]), ref["dh"]) < 2.0 ** -8 and rel(_np(out["dw"]), ref["dw"]) < 2.0 ** -8
    assert int(out["dh"].any(1).sum()) == 3


@pytest.mark.parametrize("grad", [False, True])
def test_nothing_else_is_written(grad):
    import torch
    h, w, ids, logits, t_lse, weight = _inputs(37, 72, 301, 6)
    cfg = S.DistillCfg(LS, TS, 1.0, grad)
    from paper_2607_11185_amd import _lib
    n = _lib.lib().seg_distill_workspace_bytes(37, 72, 301, 6, 0, int(grad))
    ws = torch.full((n + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    sizes = {"loss_tok": 37, "lse": 37, "loss_sum": 1, "dh": 37 * 72, "dw": 301 * 72}
    flat = {m: torch.full((s + 64,), 9.0, dtype=torch.bfloat16 if m == "dh" else torch.float32, device="cuda") for m, s in sizes.items()}
    shape = {"dh": (37, 72), "dw": (301, 72)}
    out = {m: flat[m][:s].view(shape.get(m, (s,))) for m, s in sizes.items()}
    S.seg_distill_loss(h, None, w, ids, logits, cfg, t_lse, weight, out=out, ws=ws[:n])
    want = S.seg_distill_loss(h, None, w, ids, logits, cfg, t_lse, weight)
    for m, s in sizes.items():
        if want[m] is None:
            assert bool((flat[m] == 9).all()), m
        else:
            assert torch.equal(out[m], want[m]) and bool((flat[m][s:] == 9).all()), m
    assert bool((ws[n:] == 0x5A).all())


def test_graph_streams_and_repeats():
    """Two graphs on one workspace, replayed in turn with new inputs; another stream."""
    import torch
    h, w, ids, logits, t_lse, weight = _inputs(100, 128, 2000, 20)
    cfg = S.DistillCfg(LS, TS, 1.0, True)
    ws = S.distill_workspace(100, 128, 2000, 20, 0, True, "cuda")
    out = S.seg_distill_loss(h, None, w, ids, logits, cfg, t_lse, weight, ws=ws)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            S.seg_distill_loss(h, None, w, ids, logits, cfg, t_lse, weight, out=out, ws=ws)
        graphs.append(g)
    for i in range(4):
        h.copy_(torch.randn_like(h))
        logits.copy_(torch.randn_like(logits))
        graphs[i % 2].replay()
        got = {n: t.clone() for n, t in out.items()}
        want = S.seg_distill_loss(h, None, w, ids, logits, cfg, t_lse, weight)
        assert all(torch.equal(got[n], want[n]) for n in want), i
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = S.seg_distill_loss(h, None, w, ids, logits, cfg, t_lse, weight)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(other[n], want[n]) for n in want)


def test_no_rows():
    import torch
    e = torch.empty
    out = S.seg_distill_loss(e(0, 64, device="cuda").bfloat16(), None, torch.randn(50, 64, device="cuda").bfloat16(),
                             e(0, 4, dtype=torch.int32, device="cuda"), e(0, 4, device="cuda"), S.DistillCfg(), dw_dtype=torch.bfloat16)
    assert float(out["loss_sum"]) == 0 and not bool(out["dw"].any()) and out["dh"].shape == (0, 64)


def test_from_a_teacher_in_8_bits_to_the_student():
    """The operators as they are used: a frozen teacher's projection in 8 bits, its top
    logits and their log-sum-exp, and the student's loss and gradients, beside the same
    chain in float64 from the packed values (its logits, a rounding to fp32 and 2^-12 of
    their size apart, may change which columns are the last of the top: those are taken
    from the GPU)."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(11)
    rows, hidden, vocab, k = 200, 512, 4001, 32
    x = torch.randn(rows, hidden, generator=gen, device="cuda").bfloat16()
    head = (torch.randn(vocab, hidden, generator=gen, device="cuda") * (3 / hidden ** 0.5)).bfloat16()
    h = (x.float() + 0.3 * torch.randn(rows, hidden, generator=gen, device="cuda")).bfloat16()
    w = (head.float() * 0.9).bfloat16()
    x8, head8 = S.seg_fp8_pack(x), S.seg_fp8_pack(head, 128)
    z = S.seg_fp8_gemm(x8, head8, torch.float32)
    top = S.seg_top_logits(z, k, TS)
    out = S.seg_distill_loss(h, None, w, top["ids"], top["logits"], S.DistillCfg(LS, TS, 1.0 / rows), top["lse"])
    zt = _np(S.seg_fp8_unpack(x8, torch.float32)) @ _np(S.seg_fp8_unpack(head8, torch.float32)).T
    assert rel(_np(z), zt) < 2.0 ** -12
    ids = top["ids"].cpu().numpy()
    y = zt * np.float64(np.float32(TS))
    t_lse = np.log(np.exp(y).sum(1))
    ref = OD.loss_and_grads(_bf(h), _bf(w), ids, np.take_along_axis(zt, ids.astype(np.int64), 1), np.float64(np.float32(LS)),
                            np.float64(np.float32(TS)), 1.0 / rows, t_lse)
    assert ref["p"].sum(1).max() <= 1 and ref["loss_tok"].min() > -1
    # the teacher's logits are off by 2^-12 of their size (about 3): p by that
    assert rel(_np(out["loss_tok"]), ref["loss_tok"]) < 2.0 ** -8
    assert rel(_np(out["dh"]), ref["dh"]) < 2.0 ** -7 and rel(_np(out["dw"]), ref["dw"]) < 2.0 ** -7


@pytest.mark.parametrize("rows", [3, 66])
def test_largest_vocabulary(rows):
    import torch
    vocab, hidden, k = (1 << 20) - 256, 16, 256
    gen = torch.Generator(device="cuda").manual_seed(rows)
    h = torch.randn(rows, hidden, generator=gen, device="cuda").bfloat16()
    w = torch.randn(vocab, hidden, generator=gen, device="cuda").bfloat16()
    ids = (torch.arange(k, device="cuda") * 4095 + torch.arange(rows, device="cuda")[:, None]).int().contiguous()
    ids[:, -1] = vocab - 1
    logits = torch.randn(rows, k, generator=gen, device="cuda")
    out = S.seg_distill_loss(h, None, w, ids, logits, S.DistillCfg(1.0, 1.0), dw_dtype=torch.bfloat16)
    z = h.double() @ w.double().t()
    p = torch.softmax(logits.double(), 1)
    lse = torch.logsumexp(z, 1, keepdim=True)
    loss = (p * (p.log() - torch.gather(z, 1, ids.long()) + lse)).sum(1)
    assert rel(_np(out["lse"]), _np(lse[:, 0])) < 2.0 ** -20 and rel(_np(out["loss_tok"]), _np(loss)) < 2.0 ** -18
    dz = torch.exp(z - lse).scatter_add_(1, ids.long(), -p)
    assert rel(_np(out["dh"]), _np(dz @ w.double())) < 2.0 ** -8
    assert rel(_np(out["dw"]), _np(dz.t() @ h.double())) < 2.0 ** -8


def test_weights_of_either_sign_and_scales_of_zero():
    h, w, ids, logits, t_lse, weight = _inputs(30, 64, 200, 8)
    weight[::3] *= -1
    _check(h, w, ids, logits, t_lse, weight)
    import torch
    out = S.seg_distill_loss(h, None, w, ids, logits, S.DistillCfg(0.0, 0.0, 1.0), None, weight)
    # both uniform: the student over the vocabulary, the teacher over its entries
    want = weight * float(np.log(200 / 8))
    assert bool((out["loss_tok"] - want).abs().max() < 1e-5)
    assert not bool(out["dh"].any()) and not bool(out["dw"].any())


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("rows", [9, 30, 60, 150])
def test_weights_of_nan_reach_every_row(rows, grad):
    """128 rows of the vocabulary, a whole part of the softmax's statistics, and a column of one."""
    for spoilt in (slice(128, 256), slice(290, 291)):
        h, w, ids, logits, t_lse, weight = _inputs(rows, 64, 400, 8)
        w[spoilt] = float("nan")
        ids %= 128
        weight[1] = 0
        out = S.seg_distill_loss(h, None, w, ids, logits, S.DistillCfg(1.0, 1.0, 1.0, grad), t_lse, weight)
        assert bool(out["lse"].isnan().all()) and bool(out["loss_sum"].isnan())
        assert not bool(out["loss_tok"][1].any()) and int(out["loss_tok"].isnan().sum()) == rows - 1


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("rows", [9, 30, 60, 150, 4100])
def test_rows_of_minus_infinity(rows, grad):
    """Every logit of a row is -inf: so is its log-sum-exp, as that of seg_top_logits; one
    of +inf or NaN makes it NaN.  Rows without weight stay out of all else."""
    import torch
    inf = float("inf")
    h, w, ids, logits, t_lse, weight = _inputs(rows, 64, 400, 8)
    h[:, 0], w[:, 0] = 1.0, -inf
    weight[::2] = 0
    cfg = S.DistillCfg(1.0, 1.0, 1.0, grad)
    out = S.seg_distill_loss(h, None, w, ids, logits, cfg, t_lse, weight)
    assert bool((out["lse"] == -inf).all())
    assert torch.equal(out["lse"], S.seg_top_logits(torch.full((rows, 400), -inf, device="cuda"), 1)["lse"])
    assert not bool(out["loss_tok"][::2].any()) and bool(out["loss_tok"][1::2].isnan().all())
    w[301, 0] = inf
    out = S.seg_distill_loss(h, None, w, ids, logits, cfg, t_lse, weight)
    assert bool(out["lse"].isnan().all()) and not bool(out["loss_tok"][::2].any())


@pytest.mark.parametrize("rows", [40, 100])
@pytest.mark.parametrize("what", ["id", "index", "logit", "h"])
def test_a_bad_row_reaches_the_sums(what, rows):
    """NaN in loss_tok and dh of one row; in loss_sum and all of dw, which sum over rows."""
    import torch
    h, w, ids, logits, t_lse, weight = _inputs(rows, 128, 300, 10)
    index = torch.arange(rows, device="cuda", dtype=torch.int32)
    if what == "id":
        ids[3, 2] = 300
    elif what == "index":
        index[3] = rows
    else:
        (logits if what == "logit" else h)[3, 1] = float("nan")
    out = S.seg_distill_loss(h, index, w, ids, logits, S.DistillCfg(LS, TS), t_lse, weight)
    bad = torch.arange(rows, device="cuda") == 3
    assert torch.equal(out["loss_tok"].isnan(), bad) and torch.equal(out["dh"].isnan().all(1), bad)
    assert torch.equal(out["dh"].isnan().any(1), bad)
    assert bool(out["loss_sum"].isnan()) and bool(out["dw"].isnan().all())


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("k", [5, 200])
def test_thousands_of_rows(k, given):
    """Sixteen rows a block, every one with weight but for a few: missing and repeated
    entries, and rows without weight or entries beside others."""
    import torch
    h, w, ids, logits, t_lse, weight = _inputs(4111, 64, 1003, k, given=given)
    r = torch.arange(4111, device="cuda")
    ids[r % 5 == 1, k // 2:] = -1
    ids[r % 7 == 2, 1] = ids[r % 7 == 2, 0]
    ids[r % 11 == 3, k - 1], ids[r % 11 == 3, 2] = ids[r % 11 == 3, 1], ids[r % 11 == 3, 1]
    logits[r % 13 == 4, 0] = -float("inf")
    none = (r % 17 == 5) | (r == 4110)
    weight[none] = 0
    empty = r % 19 == 6
    ids[empty] = -3
    out, _ = _check(h, w, ids, logits, t_lse, weight)
    none |= empty
    assert not bool(out["loss_tok"][none].any()) and not bool(out["dh"][none].any())
    assert bool(out["dh"][~none].any(1).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [33, 200])
def test_tensors_off_16_byte_boundaries(rows, dtype):
    """One element into their storage (w in fp32 alone, as the header asks): the same bits."""
    import torch

    def off(t):
        flat = torch.full((t.numel() + 1,), 9.0, dtype=t.dtype, device="cuda")
        flat[1:] = t.reshape(-1)
        return flat[1:].view(t.shape)

    h, w, ids, logits, t_lse, weight = _inputs(rows, 72, 301, 6, dtype=dtype)
    cfg = S.DistillCfg(LS, TS, 0.5, True)
    for dw in ("bf16", "f32"):
        want = S.seg_distill_loss(h, None, w, ids, logits, cfg, t_lse, weight, dw_dtype=_dt(dw))
        out = {n: off(t) for n, t in want.items()}
        for t in out.values():
            t.fill_(5.0)
        S.seg_distill_loss(off(h), None, off(w) if dtype == "f32" else w, off(ids), off(logits), cfg, t_lse, off(weight), out=out)
        for n, t in want.items():
            assert torch.equal(out[n], t), (n, dw)


@pytest.mark.parametrize("dw", ["bf16", "f32"])
def test_no_rows_into_any_element_of_a_buffer(dw):
    """dw one element into its storage, as calls with rows take it; nothing beside it is written."""
    import torch
    e = torch.empty
    w = torch.randn(50, 64, device="cuda").bfloat16()
    flat = torch.full((1 + 50 * 64 + 5,), 9.0, dtype=_dt(dw), device="cuda")
    out = {"loss_tok": e(0, device="cuda"), "lse": e(0, device="cuda"), "loss_sum": e(1, device="cuda"),
           "dh": e(0, 64, device="cuda").bfloat16(), "dw": flat[1:1 + 50 * 64].view(50, 64)}
    S.seg_distill_loss(e(0, 64, device="cuda").bfloat16(), None, w, e(0, 4, dtype=torch.int32, device="cuda"), e(0, 4, device="cuda"),
                       S.DistillCfg(), out=out)
    assert float(out["loss_sum"]) == 0 and not bool(out["dw"].any())
    assert float(flat[0]) == 9 and bool((flat[1 + 50 * 64:] == 9).all())


@pytest.mark.parametrize("rows", [9, 40, 150])
def test_logits_near_the_end_of_fp32(rows):
    """Sizes from 2^128 / log2(e) on count as infinite: below it they add nothing, above they are NaN."""
    import torch
    h, w, ids, logits, t_lse, weight = _inputs(rows, 64, 400, 8)
    cfg = S.DistillCfg(1.0, 1.0, 1.0, False)
    h[:, 0], w[:, 0] = 2.0 ** 64, 0.0
    want = torch.logsumexp(h.double() @ w[:140].double().t(), 1)
    w[140:, 0] = -1.36e19                                 # logits of -2.5e38, a whole part of the sums among them
    out = S.seg_distill_loss(h, None, w, ids % 140, logits, cfg, t_lse, weight)
    # fp32 sums of 64 products of about 0.25 each, and exponentials and sums as elsewhere
    assert bool(((out["lse"].double() - want).abs() <= 66 * 2.0 ** -24 * 64 + 40 * 2.0 ** -22).all())
    assert bool(out["loss_tok"].isfinite().all())
    w[:, 0] = -1.36e19
    out = S.seg_distill_loss(h, None, w, ids, logits, cfg, t_lse, weight)
    assert bool((out["lse"] == -float("inf")).all())
    w[5, 0] = 1.36e19
    out = S.seg_distill_loss(h, None, w, ids, logits, cfg, t_lse, weight)
    assert bool(out["lse"].isnan().all())
