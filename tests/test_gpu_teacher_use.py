"""The operators of a frozen teacher and its student as a training step uses them: in a
row, in a graph replayed with new inputs, from threads on streams of their own."""
import threading

import pytest

from paper_2607_11185_amd import seg as S
from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu

ROWS, MORE, HIDDEN, INTER, VOCAB, K = 150, 200, 264, 520, 5003, 24


class Step:
    """Teacher: two projections and the logits in 8 bits; student: loss and gradients."""

    def __init__(self, seed):
        import torch
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.up = S.seg_fp8_pack(self.normal(INTER, HIDDEN) * HIDDEN ** -0.5, 128)
        self.down = S.seg_fp8_pack(self.normal(HIDDEN, INTER) * INTER ** -0.5, 128)
        self.head = S.seg_fp8_pack(self.normal(VOCAB, HIDDEN) * (2 * HIDDEN ** -0.5), 128)
        self.w = (self.normal(VOCAB, HIDDEN) * (2 * HIDDEN ** -0.5)).bfloat16()
        self.index = torch.randperm(MORE, generator=self.gen, device="cuda")[:ROWS].int()
        self.weight = torch.rand(ROWS, generator=self.gen, device="cuda")
        self.weight[3] = 0
        self.x, self.h = self.normal(ROWS, HIDDEN).bfloat16(), self.normal(MORE, HIDDEN).bfloat16()

    def normal(self, *shape):
        import torch
        return torch.randn(*shape, generator=self.gen, device="cuda")

    def fresh(self):
        self.x.copy_(self.normal(ROWS, HIDDEN))
        self.h.copy_(self.normal(MORE, HIDDEN))

    def run(self):
        y = S.seg_fp8_gemm(S.seg_fp8_pack(S.seg_fp8_gemm(S.seg_fp8_pack(self.x), self.up)), self.down)
        z = S.seg_fp8_gemm(S.seg_fp8_pack(y), self.head)
        top = S.seg_top_logits(z, K, 0.8)
        out = S.seg_distill_loss(self.h, self.index, self.w, top["ids"], top["logits"], S.DistillCfg(0.9, 0.8, 1.0 / ROWS),
                                 top["lse"], self.weight)
        return [z, *top.values(), *out.values()]


def _same(a, b):
    import torch
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_step_in_plain_torch():
    """Beside the same step of elementary operations on the unpacked values: the teacher's
    product rounds to bf16 (2^-8) where that one stays in fp32, so its chosen columns are
    looked up there."""
    import torch
    s = Step(1)
    z, ids, logits, t_lse, loss, lse, total, dh, dw = s.run()
    f = lambda a: S.seg_fp8_unpack(a, torch.float32)  # noqa: E731
    again = lambda v: f(S.seg_fp8_pack(v.bfloat16()))  # noqa: E731
    want = again(again(again(s.x) @ f(s.up).t()) @ f(s.down).t()) @ f(s.head).t()
    # two packings of values a rounding apart may take neighbouring codes (2^-3 of few values)
    assert float((z.float() - want).norm() / want.norm()) < 2.0 ** -5
    best = torch.sort(z.float(), dim=1, descending=True, stable=True)
    assert torch.equal(ids, best.indices[:, :K].int()) and torch.equal(logits, best.values[:, :K])
    p = torch.exp(0.8 * logits - t_lse[:, None])
    zs = 0.9 * (s.h[s.index.long()].float() @ s.w.float().t())
    logq = zs - torch.logsumexp(zs, 1, keepdim=True)
    kl = (p * (p.log() - torch.gather(logq, 1, ids.long()))).sum(1) * s.weight
    assert float((loss - kl).norm() / kl.norm()) < 1e-4
    dz = logq.exp() * p.sum(1, keepdim=True)
    dz.scatter_add_(1, ids.long(), -p)
    dz *= (s.weight / ROWS)[:, None]
    for got, ref in ((dh, 0.9 * (dz @ s.w.float())), (dw, 0.9 * (dz.t() @ s.h[s.index.long()].float()))):
        e = float((got.float() - ref).norm() / ref.norm())
        say(e)
        assert e < 2.0 ** -8


def test_step_in_a_graph():
    """Captured twice, replayed in turn with new inputs and eager work between: the eager bits."""
    import torch
    s = Step(2)
    s.run()
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(s.run())
        graphs.append(g)
    for i in range(5):
        s.fresh()
        graphs[i % 2].replay()
        got = [t.clone() for t in outs[i % 2]]
        assert _same(got, s.run()), i
        torch.cuda.synchronize()


def test_steps_from_threads_on_their_own_streams():
    import torch
    steps = [Step(3 + i) for i in range(4)]
    want = [s.run() for s in steps]
    torch.cuda.synchronize()
    got, errors = [None] * 4, []

    def work(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(5):
                    got[i] = steps[i].run()
            stream.synchronize()
        except BaseException as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    for i in range(4):
        assert _same(got[i], want[i]), i
