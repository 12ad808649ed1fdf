"""Three-axis positions and rotation on the GPU against the float64 oracle.

Positions are integers and must be equal.  Tolerance of the rotation: angles
are reduced in fp64 and rounded to fp32 as a part of a turn in [-1/2, 1/2]
(2 pi 2^-26 = 1e-7 of a radian), sine and cosine are good to 2 ulp (2.4e-7), two
products and a sum in fp32 round three times (1.8e-7): together below 1e-6 of
|x_i| + |x_j|; a bf16 result rounds once more, by at most 2^-8 of itself."""
import numpy as np
import pytest

from oracle import layout as OL
from oracle import mrope as OM
from paper_2607_11185_amd import _lib
from paper_2607_11185_amd import seg as S
from paper_2607_11185_amd import workload as WL
from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu


def _grid(img, rng):
    """A random arrangement of every step's patches."""
    out = np.zeros((len(img), 4), np.int32)
    for s, n in enumerate(img):
        if n == 0:
            out[s] = rng.integers(-9, 9, 4)      # not looked at
            continue
        div = [k for k in range(1, n + 1) if n % k == 0]
        t = int(rng.choice(div))
        div = [k for k in range(1, n // t + 1) if n // t % k == 0]
        h = int(rng.choice(div))
        out[s] = t, h, n // t // h, rng.integers(0, 6)
    return out


def _check_positions(sp, W, L, buf=0, mode="sliding", cap=0, seed=0):
    import torch
    rng = np.random.default_rng(seed)
    grid = _grid(sp.img_len, rng)
    pr = S.Problem.from_spans(sp, W, L, cap, buf, 128, mode)
    lay = S.seg_build_layout(pr)
    n = 3 * lay.sizes.packed_tokens
    flat = torch.full((n + 999,), 12345, dtype=torch.int32, device="cuda")
    pos = flat[:n].view(3, -1)
    S.seg_mrope_positions(pr, lay, grid, pos)
    assert bool((flat[n:] == 12345).all())
    ref = OL.build(sp, W, L, 128, cap=cap, buffer_tokens=buf, with_tiles=False, mode=mode)
    want = OM.positions(ref, sp, grid, ref.packed_tokens)
    say(f"positions: {lay.sizes.packed_tokens} rows, {lay.sizes.num_segments} segments")
    bad = np.argwhere(pos.cpu().numpy() != want)
    assert len(bad) == 0, (len(bad), bad[:3].tolist())


@pytest.mark.parametrize("name,kw", [
    ("one_row", dict(turns=[1], prompt=[1], img=[0], text=[0], act=[0], W=1, L=1)),
    ("no_text", dict(turns=[3], prompt=[0], img=[6, 1, 12], text=[0, 0, 1], act=[0, 0, 1], W=2, L=3)),
    ("ragged", dict(turns=[3, 0, 5], prompt=[5, 9, 1], img=[7, 0, 30, 12, 0, 0, 2047, 36], text=[1, 2, 0, 700, 3, 1025, 1, 9],
                    act=[1, 0, 0, 5, 1, 2, 1, 1], W=2, L=2)),
    ("buffers", dict(turns=[4, 4], prompt=[8, 3], img=[24] * 8, text=[5, 6, 7, 8, 9, 1, 2, 3], act=[1] * 8, W=2, L=2, buf=1111)),
    ("anchored", dict(turns=[7], prompt=[8], img=[60, 48, 36, 30, 24, 12, 8], text=[5] * 7, act=[1] * 7, W=2, L=2,
                      mode="anchored"))])
def test_positions(name, kw):
    say(name)
    sp = WL.explicit_spans(kw["turns"], kw["prompt"], kw["img"], kw["text"], kw["act"])
    _check_positions(sp, kw["W"], kw["L"], kw.get("buf", 0), kw.get("mode", "sliding"))


def test_positions_of_many_short_runs():
    """Runs of one to three rows, many to a block of rows, with screenshots and without."""
    rng = np.random.default_rng(9)
    n = 900
    sp = WL.explicit_spans([n], [1], rng.choice([0, 1, 2, 3], n), rng.integers(1, 3, n), [0] * n)
    _check_positions(sp, n, n)
    _check_positions(sp, 40, 300, buf=4096)


@pytest.mark.parametrize("seed", range(6))
def test_positions_random(seed):
    rng = np.random.default_rng(100 + seed)
    T = rng.integers(0, 9, size=4)
    ns = int(T.sum())
    text = rng.integers(0, 300, size=ns)
    sp = WL.explicit_spans(T, rng.integers(1, 9, size=4), rng.integers(0, 3, size=ns) * rng.integers(1, 200, size=ns), text,
                           [int(rng.integers(0, min(t, 5) + 1)) for t in text])
    _check_positions(sp, int(rng.integers(1, 4)), int(rng.integers(1, 5)), int(rng.choice([0, 9000])),
                     "anchored" if seed % 3 == 2 else "sliding", seed=seed)


def test_positions_of_an_empty_problem():
    pr = S.Problem.from_spans(WL.explicit_spans([], [], [], [], []), 1, 1)
    lay = S.seg_build_layout(pr)
    assert S.seg_mrope_positions(pr, lay, None).shape == (3, 0)


def _rows(rows, heads, d, dt, stride_heads=0, offset=0, gen=None):
    """[rows, heads, d], as a part of wider rows where stride_heads says so."""
    import torch
    base = torch.randn(rows, max(heads, stride_heads), d, generator=gen, device="cuda").to(dt)
    return base[:, offset:offset + heads]


def _bound(x, ref, dt):
    import torch
    half = x.shape[-1] // 2
    mag = np.abs(x[..., :half]) + np.abs(x[..., half:])
    tol = 1e-6 * np.concatenate([mag, mag], -1)
    return tol + (2.0 ** -8 * (np.abs(ref) + tol) if dt == torch.bfloat16 else 0)


CASES = [(1, 28, 4, 128, (16, 24, 24)), (1, 1, 0, 16, (0, 0, 8)), (3, 5, 1, 48, (7, 11, 6)), (257, 12, 4, 64, (8, 12, 12)),
         (1000, 16, 2, 128, (64, 0, 0)), (77, 2, 2, 256, (1, 63, 64)), (130, 3, 1, 96, (0, 48, 0)), (65, 40, 0, 16, (3, 2, 3)),
         (5, 200, 8, 128, (16, 24, 24))]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c[:4])))
def test_rotation(case, dtype):
    import torch
    rows, hq, hkv, d, sections = case
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(rows)
    pos = torch.randint(0, 1 << 20, (3, rows), generator=gen, device="cuda", dtype=torch.int32)
    if rows > 2:
        pos[0, 1] = -1
        pos[2, rows - 1] = -1
    pos[0, 0] = 0
    if rows > 4:
        pos[1, 4] = 2 ** 31 - 1                  # an angle of 2^31 radians
    cfg = S.MropeCfg(sections, 1e4)
    q = _rows(rows, hq, d, dt, hq + 3, 2, gen)
    k = _rows(rows, hkv, d, dt, hkv + 1, 1, gen) if hkv else None
    pn = pos.cpu().numpy()
    for f, inverse in ((S.seg_mrope_fwd, False), (S.seg_mrope_bwd, True)):
        qo = torch.full((rows + 3, hq + 1, d), 7.0, dtype=dt, device="cuda")
        got = f(q, k, pos, cfg, qo[:rows, :hq])
        assert bool((qo[rows:] == 7.0).all())
        for x, y in zip((q, k), got):
            if x is None:
                assert y is None
                continue
            xn = x.double().cpu().numpy()
            ref = OM.rotate(xn, pn, sections, 1e4, inverse)
            err = np.abs(y.double().cpu().numpy() - ref)
            # fp64 angles near 2^31 are good to 2^31 2^-53 (a few roundings): 1e-6
            far = np.where((pn > 1 << 20).any(0), 2e-6, 0.0)[:, None, None] * np.abs(xn).max()
            over = err - _bound(xn, ref, dt) - far
            worst = float(over.max())
            assert worst <= 0, (case, dtype, inverse, worst)
        assert bool((qo[:, hq] == 7.0).all())    # what lies between the rows and behind them is left alone


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotation_in_place_and_back(dtype):
    """In place equals out of place bit for bit; turning back undoes it (fp32: two rotations,
    1e-6 of the pair each)."""
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(5)
    qkv = _rows(333, 8, 64, dt, gen=gen)
    pos = torch.randint(0, 40000, (3, 333), generator=gen, device="cuda", dtype=torch.int32)
    pos[:, 100] = -1
    cfg = S.MropeCfg((8, 12, 12))
    want = S.seg_mrope_fwd(qkv[:, :4], qkv[:, 4:6], pos, cfg)
    copy = qkv.clone()
    got = S.seg_mrope_fwd(copy[:, :4], copy[:, 4:6], pos, cfg, copy[:, :4], copy[:, 4:6])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(copy[:, 6:], qkv[:, 6:]) and torch.equal(copy[100], qkv[100])
    back = S.seg_mrope_bwd(*want, pos, cfg)
    assert not back[0][100].any() and not back[1][100].any()
    if dtype == "f32":
        ok = torch.arange(333, device="cuda") != 100
        assert float((back[0] - qkv[:, :4])[ok].abs().max()) <= 4e-6 * float(qkv.abs().max())


def test_rotation_transpose():
    """<R x, y> = <x, R^T y> in fp32 (both sums in fp64; 1e-6 of each pair)."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(6)
    x, y = (_rows(129, 6, 128, torch.float32, gen=gen) for _ in range(2))
    pos = torch.randint(0, 100000, (3, 129), generator=gen, device="cuda", dtype=torch.int32)
    cfg = S.MropeCfg((16, 24, 24))
    a = (S.seg_mrope_fwd(x, None, pos, cfg)[0].double() * y.double()).sum()
    b = (x.double() * S.seg_mrope_bwd(y, None, pos, cfg)[0].double()).sum()
    assert abs(float(a - b)) <= 4e-6 * float((x.abs().double() * y.abs().double()).sum() * 2)


def test_rotation_nonfinite_and_empty():
    import torch
    x = torch.ones(2, 1, 16, device="cuda")
    x[0, 0, 3] = float("inf")
    x[1, 0, 11] = float("nan")
    pos = torch.tensor([[0, -1]] * 3, dtype=torch.int32, device="cuda")
    y, _ = S.seg_mrope_fwd(x, None, pos, S.MropeCfg((8, 0, 0), 1e4))
    assert torch.isnan(y[0, 0, 11]) and torch.isinf(y[0, 0, 3])   # inf times sin 0
    assert torch.equal(y[1].nan_to_num(3.0), x[1].nan_to_num(3.0))
    assert not S.seg_mrope_bwd(x, None, pos, S.MropeCfg((8, 0, 0), 1e4))[0][1].any()
    empty = torch.empty(0, 4, 64, device="cuda")
    assert S.seg_mrope_fwd(empty, empty, pos[:, :0].contiguous(), S.MropeCfg((32, 0, 0)))[0].shape == (0, 4, 64)


def test_rotation_refuses_unaligned_rows_before_any_launch():
    import torch
    x = torch.zeros(4 * 70 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(4, 1, 70)[:, :, :64]
    pos = torch.zeros((3, 4), dtype=torch.int32, device="cuda")
    with pytest.raises(_lib.SegError) as e:
        S.seg_mrope_fwd(x, None, pos, S.MropeCfg((32, 0, 0)))
    assert e.value.status == _lib.SEG_ERR_UNSUPPORTED
    with pytest.raises(AssertionError):
        S.seg_mrope_fwd(x.cpu(), None, pos, S.MropeCfg((32, 0, 0)))


def test_rotation_with_positions_between_the_rows():
    """Positions that lie in the gap behind an output's first or last row share nothing with it."""
    import torch
    q = torch.randn(4, 2, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(8))
    pos = torch.randint(0, 1000, (3, 4), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(9))
    cfg = S.MropeCfg((8, 12, 12))
    want = S.seg_mrope_fwd(q, None, pos, cfg)[0]
    for row in (0, 3):
        buf = torch.zeros(4, 256, device="cuda")
        here = buf[row, 128:140].view(torch.int32).view(3, 4)
        here.copy_(pos)
        got = S.seg_mrope_fwd(q, None, here, cfg, buf[:, :128].view(4, 2, 64))[0]
        assert torch.equal(got, want) and torch.equal(here, pos)


@pytest.mark.parametrize("inverse", [False, True])
def test_rotation_near_a_quarter_turn(inverse):
    """Angles whose cosine or sine is close to zero, fp32: x = (1, 0) turns to (cos, sin), each
    good relative to itself: 2 ulp of the sine and cosine and one rounding (2.5 ulp), besides the
    fp64 angle (160 turns, 14 bits of exponent: 3e-12 of a radian, 1e-11 with room)."""
    import torch
    rows, d, base = 1001, 64, 1e4
    pos = np.arange(rows)
    x = torch.zeros(rows, 1, d, device="cuda")
    x[..., :d // 2] = 1
    p = torch.from_numpy(np.stack([pos] * 3).astype(np.int32)).cuda()
    f = S.seg_mrope_bwd if inverse else S.seg_mrope_fwd
    got = f(x, None, p, S.MropeCfg((d // 2, 0, 0), base))[0][:, 0].double().cpu().numpy()
    ref = OM.rotate(x.double().cpu().numpy(), np.stack([pos] * 3), (d // 2, 0, 0), base, inverse)[:, 0]
    assert (np.abs(ref[pos > 0]) < 1e-3).sum() > 20
    over = np.abs(got - ref) - 2.5 * 2.0 ** -23 * np.abs(ref) - 1e-11
    assert over.max() <= 0, (float(over.max()), int((over > 0).sum()))


@pytest.mark.parametrize("dtype,rows", [("f32", 20011), ("bf16", 40013)])
@pytest.mark.parametrize("inverse", [False, True])
def test_rotation_past_the_caches(dtype, rows, inverse):
    """Tensors of more than 96 MB read and written, in place and not: every row as in calls of a
    few rows."""
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(rows)
    qkv = _rows(rows, 14, 64, dt, gen=gen)
    pos = torch.randint(-20, 100000, (3, rows), generator=gen, device="cuda", dtype=torch.int32)
    cfg = S.MropeCfg((8, 12, 12))
    f = S.seg_mrope_bwd if inverse else S.seg_mrope_fwd
    assert 2 * rows * 13 * 64 * qkv.element_size() > 96 << 20
    say(f"{rows} x 13 x 64 {dtype}")
    got = f(qkv[:, :12], qkv[:, 12:13], pos, cfg)
    for r in range(0, rows, 5000):
        s = slice(r, min(r + 5000, rows))
        want = f(qkv[s, :12], qkv[s, 12:13], pos[:, s].contiguous(), cfg)
        assert torch.equal(got[0][s], want[0]) and torch.equal(got[1][s], want[1]), s
    copy = qkv.clone()
    f(copy[:, :12], copy[:, 12:13], pos, cfg, copy[:, :12], copy[:, 12:13])
    assert torch.equal(copy[:, :12], got[0]) and torch.equal(copy[:, 12:13], got[1]) and torch.equal(copy[:, 13:], qkv[:, 13:])
