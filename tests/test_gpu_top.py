"""Selection of the largest logits on the GPU: columns and values equal the float64
oracle's exactly; the log-sum-exp within the fp32 evaluation's bound.

With y = scale z rounded once (2^-24 |y|) and m the largest: an exponent y - m rounds
(2^-24 |y - m|) and again as a product by log2(e) (2^-24 of its size, and log2(e)'s own
rounding), the exponential is good to 2^-22, so a term e^x of x = y - m is off by (4 |x|
+ 4 + |y|) 2^-24 of itself; |x| e^x sums to at most the sum times log(n) + 1 (entropy).
The sum of n terms, in lanes of a few hundred and then a tree, and its rescaling by
exp(old m - new m) at every step of eight columns, round n / 256 + 100 times.  So lse is
off by at most ((4 log n + 8) + |y|max + n / 128 + 200) 2^-24, and 2^-24 |lse| for its
last sum."""
import numpy as np
import pytest

from oracle import top as OT
from paper_2607_11185_amd import _lib
from paper_2607_11185_amd import seg as S
from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu


def _dt(name):
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def _check(z, k, scale=1.0):
    got = S.seg_top_logits(z, k, scale)
    zn = z.double().cpu().numpy()
    ids, values = OT.top(zn, k)
    g = got["ids"].cpu().numpy()
    assert np.array_equal(g, ids), np.argwhere(g != ids)[:5]
    v = got["logits"].double().cpu().numpy()
    assert np.array_equal(v, values, equal_nan=True)
    want, lse = OT.lse(zn, np.float64(np.float32(scale))), got["lse"].double().cpu().numpy()
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(lse)) and np.array_equal(want[~fine], lse[~fine], equal_nan=True)
    if fine.any():
        y = np.abs(np.where(np.isfinite(zn), zn, 0)).max(1) * abs(scale)
        n = z.shape[1]
        tol = ((4 * np.log(n) + 8) + y + n / 128 + 200) * 2.0 ** -24 + 2.0 ** -24 * np.abs(want, where=fine, out=np.zeros_like(want))
        assert bool((np.abs(want - lse)[fine] <= tol[fine]).all())
    return got


def _z(rows, vocab, dtype, seed=0, std=2.5):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed * 100 + rows + vocab)
    return (torch.randn(rows, vocab, generator=gen, device="cuda") * std).to(_dt(dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab,k", [(1, 1, 1), (2, 5, 5), (3, 63, 20), (4, 64, 64), (2, 65, 7), (5, 256, 256), (3, 1001, 1),
                                          (7, 1001, 200), (2, 16384, 256), (3, 16385, 256), (37, 32000, 64), (1, 151936, 20),
                                          (2, 151936, 256), (300, 5003, 33), (1, 1 << 20, 50), (3, 300000, 100),
                                          # without groups, and a block a row with them
                                          (4, 4096, 256), (3, 4097, 70), (2, 16384, 1), (5, 12000, 255), (530, 4500, 40), (530, 16384, 256),
                                          (600, 4000, 16), (70, 5000, 9), (64, 65536, 32), (66, 65537, 32), (63, 20000, 100),
                                          (512, 40, 7), (600, 1001, 33), (515, 5000, 256), (700, 2048, 1), (513, 20001, 64)])
def test_columns_and_values(rows, vocab, k, dtype):
    say(rows, vocab, k, dtype)
    _check(_z(rows, vocab, dtype), k)


@pytest.mark.parametrize("scale", [0.5, 1.7, 0.0, -1.3])
def test_scale(scale):
    _check(_z(9, 3000, "bf16"), 11, scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab,wide,at", [(4096, 4200, 8), (4096, 4103, 3), (1000, 1001, 1)])
def test_parts_of_wider_rows(vocab, wide, at, dtype):
    _check(_z(33, wide, dtype)[:, at:at + vocab], 40)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [9, 540])
@pytest.mark.parametrize("vocab,k", [(40000, 64), (40000, 256), (700, 256), (100, 9), (151936, 3)])
def test_orders_and_ties(vocab, k, rows, dtype):
    """All alike; two values; ascending and descending; ties across groups; both zeros."""
    import torch
    if rows * vocab > 1 << 25:
        rows = 9
    z = torch.zeros(rows, vocab, device="cuda")
    n = torch.arange(vocab, device="cuda").float()
    z[0] = 1.25
    z[1] = (n % 2)
    z[2] = n / vocab
    z[3] = -n / vocab
    z[4] = torch.where(n % 2 == 0, -0.0, 0.0)
    z[5] = (n % 97).floor()
    z[6] = -7.0
    z[6, -1] = 3.0
    z[7] = torch.where(n < vocab // 2, 5.0, 5.0)
    z[7, 3] = 4.0
    z[8] = -torch.where(n % 3 == 0, 0.0, 1.0)
    _check(z.to(_dt(dtype)), k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masks_infinities_and_nan(dtype):
    import torch
    low = torch.finfo(_dt(dtype)).min
    z = _z(10, 5000, dtype)
    z[0] = -float("inf")
    z[1, 10:] = -float("inf")                # fewer numbers than k
    z[2] = low
    z[3, 5:] = low
    z[4, 4000] = float("inf")
    z[5, 4999], z[5, 77] = float("nan"), float("nan")
    z[6, 1], z[6, 2], z[6, 3] = float("inf"), float("nan"), -float("inf")
    z[7, ::2] = -float("inf")
    z[8] = float("nan")
    z[9] = float("inf")
    _check(z, 40)
    _check(z, 256)


def test_past_32_bits():
    """Rows behind 2^31 elements."""
    import torch
    z = torch.full((15000, 151936), -1.0, dtype=torch.bfloat16, device="cuda")
    z[14999, 151000], z[14999, 5], z[14200, 7] = 3.0, 2.0, 1.0
    got = S.seg_top_logits(z, 3)
    assert got["ids"][14999].tolist() == [151000, 5, 0] and got["logits"][14999].tolist() == [3.0, 2.0, -1.0]
    assert got["ids"][14200].tolist() == [7, 0, 1]
    assert got["ids"][0].tolist() == [0, 1, 2]


@pytest.mark.parametrize("rows,vocab,k", [(3, 5000, 20), (2, 100, 100)])
def test_nothing_else_is_written(rows, vocab, k):
    import torch
    z = _z(rows, vocab, "bf16")
    n = _lib.lib().seg_top_logits_workspace_bytes(rows, vocab)
    ws = torch.full((n + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    flat = {"ids": torch.full((rows * k + 64,), 9, dtype=torch.int32, device="cuda"),
            "logits": torch.full((rows * k + 64,), 9.0, device="cuda"), "lse": torch.full((rows + 64,), 9.0, device="cuda")}
    out = {"ids": flat["ids"][:rows * k].view(rows, k), "logits": flat["logits"][:rows * k].view(rows, k), "lse": flat["lse"][:rows]}
    S.seg_top_logits(z, k, out=out, ws=ws[:n])
    want = S.seg_top_logits(z, k)
    for name, t in flat.items():
        assert torch.equal(out[name], want[name])
        assert bool((t[want[name].numel():] == 9).all())
    assert bool((ws[n:] == 0x5A).all())


def test_graph_streams_and_repeats():
    import torch
    z = _z(50, 20000, "f32")
    ws = S.top_logits_workspace(50, 20000, "cuda")
    out = S.seg_top_logits(z, 33, ws=ws)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):                                   # one workspace in two graphs
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            S.seg_top_logits(z, 33, out=out, ws=ws)
        graphs.append(g)
    for i in range(4):
        z.copy_(torch.randn_like(z))
        graphs[i % 2].replay()
        got = {n: t.clone() for n, t in out.items()}
        want = S.seg_top_logits(z, 33)
        assert all(torch.equal(got[n], want[n]) for n in want), i
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = S.seg_top_logits(z, 33)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(other[n], want[n]) for n in want)


def test_no_rows():
    import torch
    got = S.seg_top_logits(torch.empty(0, 50, device="cuda"), 5)
    assert got["ids"].shape == (0, 5) and got["lse"].shape == (0,)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab,k", [(3000, 3000, 40), (1500, 9000, 200), (2500, 20000, 50), (40, 300000, 64), (40, 70000, 256)])
def test_many_rows_of_one_value(rows, vocab, k, dtype):
    """Two searches behind each other in every block, the first of which has nothing to cut."""
    import torch
    z = torch.arange(rows, device="cuda", dtype=torch.float32)[:, None].expand(rows, vocab).to(_dt(dtype)).contiguous()
    first = torch.arange(k, device="cuda", dtype=torch.int32).expand(rows, k)
    for _ in range(4):
        got = S.seg_top_logits(z, k)
        assert torch.equal(got["ids"], first) and torch.equal(got["logits"], z[:, :k].float())


@pytest.mark.parametrize("scale", [1.0, -0.7])
@pytest.mark.parametrize("k", [64, 256])
@pytest.mark.parametrize("rows,vocab,wide,dtype", [(1700, 32003, 32003, "bf16"), (1700, 32003, 32010, "bf16"), (800, 33001, 33001, "f32"),
                                                   (530, 151933, 151936, "bf16")])
def test_logits_past_the_caches(rows, vocab, wide, dtype, k, scale):
    """More than 96 MB, read past the caches: columns, values and log-sum-exp against torch in
    64 bits (a stable sort has ties in the order of their columns)."""
    import torch
    z = _z(rows, wide, dtype)[:, :vocab]
    z[3, 17], z[4, 5:], z[5, vocab - 1] = -float("inf"), -float("inf"), 30.0
    z[7, 9], z[8] = float("nan"), -float("inf")
    got = S.seg_top_logits(z, k, scale)
    for at in range(0, rows, 200):
        part = z[at:at + 200].double()
        # (NaN sorts as the largest; -0 as 0)
        value, column = torch.sort(part + 0.0, dim=1, descending=True, stable=True)
        assert torch.equal(got["ids"][at:at + 200], column[:, :k].int())
        assert torch.equal(got["logits"][at:at + 200].double().nan_to_num(7.0, 8.0, 9.0), value[:, :k].nan_to_num(7.0, 8.0, 9.0))
        y = part * float(np.float32(scale))
        want, lse = torch.logsumexp(y, 1), got["lse"][at:at + 200].double()
        fine = want.isfinite()
        assert torch.equal(fine, lse.isfinite())
        assert torch.equal(want[~fine].nan_to_num(7.0, 8.0, 9.0), lse[~fine].nan_to_num(7.0, 8.0, 9.0))
        tol = ((4 * np.log(vocab) + 8) + torch.where(y.isfinite(), y, 0).abs().amax(1) + vocab / 128 + 200) * 2.0 ** -24 + 2.0 ** -24 * want.abs()
        assert bool(((want - lse).abs() <= tol)[fine].all())


def test_sums_past_32_bits():
    """Rows of one value each, behind 2^31 elements: its log-sum-exp is value + log(vocab)."""
    import torch
    rows, vocab = 15000, 151936
    value = (torch.arange(rows, device="cuda") % 9 - 4).bfloat16()
    got = S.seg_top_logits(value[:, None].expand(rows, vocab).contiguous(), 2, 0.5)
    want = value.double() * 0.5 + float(np.log(vocab))
    tol = ((4 * np.log(vocab) + 8) + 2 + vocab / 128 + 200) * 2.0 ** -24 + 2.0 ** -24 * want.abs()
    assert bool(((got["lse"].double() - want).abs() <= tol).all())
    assert torch.equal(got["logits"], value[:, None].float().expand(rows, 2))
