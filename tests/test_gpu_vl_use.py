"""The operators as programs use them: on streams of their own, two at once, with one
workspace in two captured graphs, over tensors whose elements pass 2^32."""
import pytest

from paper_2607_11185_amd import seg as S
from tests.gpu_helpers import rel, say

pytestmark = pytest.mark.gpu


def _gen(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


def _work(seed, rows=700):
    """Inputs and a call sequence over them: rotation, packing, the gated block and its backward."""
    import torch
    g = _gen(seed)
    qk = torch.randn(rows, 6, 64, generator=g, device="cuda").to(torch.bfloat16)
    pos = torch.randint(0, 5000, (3, rows), generator=g, device="cuda", dtype=torch.int32)
    x = torch.randn(rows, 256, generator=g, device="cuda").to(torch.bfloat16)
    w = [torch.randn(1032, 256, generator=g, device="cuda").div(16).to(torch.bfloat16) for _ in range(2)]
    dm = torch.randn(rows, 1032, generator=g, device="cuda").to(torch.bfloat16)

    def run():
        q, k = S.seg_mrope_fwd(qk[:, :4], qk[:, 4:], pos, S.MropeCfg((8, 12, 12)))
        xv = S.seg_act_unpack(S.seg_act_pack(x))
        m, kept = S.seg_glu_fwd(xv, *w, keep=True)
        out = S.seg_glu_bwd(xv, *w, dm, kept)
        return [q, k, xv, m, kept[0].code, kept[0].exp, kept[1].code, kept[1].exp, *out.values()]
    return run


def test_two_streams_at_once():
    import torch
    runs = [_work(1), _work(2, 333)]
    want = [r() for r in runs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for rep in range(3):
        got = [None, None]
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                got[i] = runs[i]()
        for s in streams:
            s.synchronize()
        for i in (0, 1):
            assert all(torch.equal(a, b) for a, b in zip(got[i], want[i])), (rep, i)


def test_calls_from_two_threads():
    import threading

    import torch
    runs = [_work(3), _work(4, 65)]
    want = [r() for r in runs]
    torch.cuda.synchronize()
    bad = []

    def work(i):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(5):
                got = runs[i]()
                s.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want[i])):
                    bad.append(i)
    ts = [threading.Thread(target=work, args=(i,)) for i in (0, 1)]
    for t in ts:
        t.start()
    for t in ts:
        t.join(60)
    assert not bad


def test_one_workspace_in_two_graphs():
    """A forward whose product is cut over K, and a backward, captured in a graph each with the
    same workspace and replayed in turns."""
    import torch
    g = _gen(5)
    x = torch.randn(300, 1024, generator=g, device="cuda").to(torch.bfloat16)
    w = [torch.randn(264, 1024, generator=g, device="cuda").div(32).to(torch.bfloat16) for _ in range(2)]
    dm = torch.randn(300, 264, generator=g, device="cuda").to(torch.bfloat16)
    m, kept = S.seg_glu_fwd(x, *w, keep=True)
    want_m, want = m.clone(), {n: t.clone() for n, t in S.seg_glu_bwd(x, *w, dm, kept).items()}
    n = max(S.glu_workspace(300, 1024, 264, b, True, "cuda").numel() for b in (False, True))
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    kept2 = (S.Act8.empty(300, 264, "cuda"), S.Act8.empty(300, 264, "cuda"))
    out = {k: torch.empty_like(t) for k, t in want.items()}
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    with torch.cuda.graph(graphs[0]):
        S.seg_glu_fwd(x, *w, keep=kept2, m=m, ws=ws)
    with torch.cuda.graph(graphs[1]):
        S.seg_glu_bwd(x, *w, dm, kept2, out=out, ws=ws)
    for rep in range(3):
        for t in (m, kept2[0].code, kept2[1].exp, *out.values()):
            t.fill_(3)
        ws.fill_(255)
        torch.cuda.synchronize()
        graphs[0].replay()
        graphs[1].replay()
        graphs[0].replay()
        torch.cuda.synchronize()
        assert torch.equal(m, want_m) and torch.equal(kept2[0].code, kept[0].code) and torch.equal(kept2[1].exp, kept[1].exp)
        assert all(torch.equal(out[k], want[k]) for k in want), rep


def _parts(rows, at):
    """Slices of rows at the start, around row `at` and at the end."""
    return [slice(0, 64), slice(at - 40, at + 40), slice(rows - 70, rows)]


def test_packing_past_32_bit_offsets():
    import torch
    rows, cols = 1300000, 3584
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda").normal_(generator=_gen(6))
    say(f"{x.numel() / 2 ** 32:.2f} x 2^32 elements")
    p = S.seg_act_pack(x)
    back = S.seg_act_unpack(p)
    for s in _parts(rows, 2 ** 32 // cols):
        q = S.seg_act_pack(x[s])
        assert torch.equal(p.code[s], q.code) and torch.equal(p.exp[s], q.exp)
        assert torch.equal(back[s], S.seg_act_unpack(q))


def test_rotation_past_32_bit_offsets():
    import torch
    rows = 1100000
    qkv = torch.empty(rows, 36, 128, dtype=torch.bfloat16, device="cuda").normal_(generator=_gen(7))
    pos = torch.randint(0, 100000, (3, rows), generator=_gen(8), device="cuda", dtype=torch.int32)
    cfg = S.MropeCfg((16, 24, 24))
    q, k = S.seg_mrope_fwd(qkv[:, :28], qkv[:, 28:32], pos, cfg)
    for s in _parts(rows, 2 ** 32 // (36 * 128)):
        a, b = S.seg_mrope_fwd(qkv[s, :28], qkv[s, 28:32], pos[:, s].contiguous(), cfg)
        assert torch.equal(q[s], a) and torch.equal(k[s], b)


def test_gated_block_past_32_bit_offsets():
    """K is one step of the products here, so a row of the forward has one order of summing
    whatever the number of rows: equal to a call on a part of the rows.  dx sums over 2 x 4,104
    values in parts that depend on it: two roundings of 2^-8 of dg and du, and of dx."""
    import torch
    rows, hidden, inter = 1 << 20, 64, 4104
    x = torch.empty(rows, hidden, dtype=torch.bfloat16, device="cuda").normal_(generator=_gen(9))
    w = [torch.empty(inter, hidden, dtype=torch.bfloat16, device="cuda").normal_(std=0.15, generator=_gen(10 + i)) for i in (0, 1)]
    m, kept = S.seg_glu_fwd(x, *w, keep=True)
    dm = torch.empty_like(m).normal_(generator=_gen(12))
    out = S.seg_glu_bwd(x, *w, dm, kept)
    for s in [slice(0, 300), slice(2 ** 32 // inter - 200, 2 ** 32 // inter + 100), slice(rows - 300, rows)]:
        ms, ks = S.seg_glu_fwd(x[s], *w, keep=True)
        assert torch.equal(m[s], ms)
        for a, b in zip(kept, ks):
            assert torch.equal(a.code[s], b.code) and torch.equal(a.exp[s], b.exp)
        os_ = S.seg_glu_bwd(x[s], *w, dm[s], ks)
        assert torch.equal(out["m"][s], os_["m"])
        assert rel(out["dx"][s].double().cpu().numpy(), os_["dx"].double().cpu().numpy()) < 2.0 ** -8
