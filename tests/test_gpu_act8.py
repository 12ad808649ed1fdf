"""8-bit activations on the GPU: codes, exponent bytes and values equal the
float64 oracle's exactly (scaling by a power of two rounds nothing, so the one
rounding is to the nearest integer)."""
import numpy as np
import pytest

from oracle import act8 as OA8
from paper_2607_11185_amd import seg as S
from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu


def _same(got, want, what):
    """Equal as numbers (NaN with NaN); says where they are not."""
    got = got.cpu().numpy() if hasattr(got, "cpu") else got
    bad = np.argwhere(~((got == want) | (np.isnan(got) & np.isnan(want))) if got.dtype.kind == "f" else got != want)
    if got.shape != want.shape or len(bad):
        at = tuple(bad[0])
        raise AssertionError(f"{what}: {len(bad)} differ, first at {at}: {got[at]}, not {want[at]}")


def _check(x):
    """x [rows, cols] on the GPU, perhaps a part of wider rows."""
    import torch
    got = S.seg_act_pack(x)
    code, exp = OA8.pack(x.double().cpu().numpy())
    _same(got.exp, exp, "exponents")
    _same(got.code, code, "codes")
    want = OA8.unpack(code, exp)
    for dt in (torch.bfloat16, torch.float32):
        _same(S.seg_act_unpack(got, dt).double(), want, f"values in {dt}")
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (3, 31), (2, 32), (5, 33), (7, 100), (4, 264), (33, 1001), (9, 2048),
                                       (301, 3584), (1000, 40), (2, 18944), (4099, 8)])
def test_codes_and_values(rows, cols, dtype):
    import torch
    say(f"{rows} x {cols} {dtype}")
    gen = torch.Generator(device="cuda").manual_seed(rows * 7 + cols)
    x = torch.randn(rows, cols, generator=gen, device="cuda")
    x *= torch.exp(4 * torch.randn(rows, 1, generator=gen, device="cuda"))      # rows of any size
    x[torch.rand(rows, cols, generator=gen, device="cuda") < 0.1] = 0
    if rows > 3:
        x[2] = 0
    _check(x.to(torch.bfloat16 if dtype == "bf16" else torch.float32))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cols,wide,at", [(96, 128, 16), (96, 100, 4), (100, 131, 3), (64, 65, 1)])
def test_parts_of_wider_rows(cols, wide, at, dtype):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(cols)
    base = torch.randn(37, wide, generator=gen, device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    x = base[:, at:at + cols]
    got = _check(x)
    out = torch.full_like(base, 7.0)
    S.seg_act_unpack(got, x=out[:, at:at + cols])
    keep = torch.ones(wide, dtype=torch.bool, device="cuda")
    keep[at:at + cols] = False
    assert bool((out[:, keep] == 7.0).all())
    assert torch.equal(out[:, at:at + cols], S.seg_act_unpack(got, base.dtype))


def test_borders_of_a_block():
    """Ties, the largest code, a step more, the smallest and largest numbers of fp32, and
    what is not finite."""
    import torch
    inf, nan = float("inf"), float("nan")
    top = float(np.finfo(np.float32).max)
    blocks = [[127.0, 2.5, 3.5, -0.5, -1.5, 126.5], [np.nextafter(np.float32(127), np.float32(200)), 1.0, 3.0], [63.5, 63.25, 0.25],
              [top, -top, top / 3, 1.0], [1e-45, -1e-45, 3e-45], [2.0 ** -126, 2.0 ** -127, -2.0 ** -133], [0.0, -0.0],
              [inf, 1.0], [1.0, -inf], [nan, 5.0], [-nan, inf, 0.0], [2.0 ** -120, 2.0 ** -149], [-127.0, 127.0]]
    x = torch.zeros(len(blocks), 64, device="cuda")
    for i, b in enumerate(blocks):
        x[i, 32 * (i % 2):32 * (i % 2) + len(b)] = torch.tensor(b)
    got = _check(x)
    assert sorted(set(got.exp.flatten().tolist()))[-1] == 255
    bad = ~torch.isfinite(x).view(-1, 2, 32).all(-1)
    v = S.seg_act_unpack(got, torch.float32).view(-1, 2, 32)
    assert bool(torch.isnan(v[bad]).all()) and bool(torch.isfinite(v[~bad]).all())
    _check(x.to(torch.bfloat16))


def test_values_are_kept_by_a_second_packing():
    import torch
    x = torch.randn(50, 200, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    v = S.seg_act_unpack(S.seg_act_pack(x), torch.float32)
    assert torch.equal(S.seg_act_unpack(S.seg_act_pack(v), torch.float32), v)
    # at most half a step, a step being at most 2 / 127 of the block's largest magnitude
    top = torch.nn.functional.pad(x.abs(), (0, 24)).view(50, -1, 32).amax(-1).repeat_interleave(32, 1)[:, :200]
    assert bool(((v - x).abs() <= top / 127).all())


def test_empty():
    import torch
    x = torch.empty(0, 40, device="cuda")
    assert S.seg_act_unpack(S.seg_act_pack(x), torch.float32).shape == (0, 40)


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 31), (7, 100), (33, 1001), (301, 3584)])
def test_nothing_is_written_past_the_end(rows, cols):
    import torch
    x = torch.randn(rows, cols, device="cuda")
    code = torch.full((rows * cols + 999,), 77, dtype=torch.int8, device="cuda")
    nb = -(-cols // 32)
    exp = torch.full((rows * nb + 999,), 77, dtype=torch.uint8, device="cuda")
    out = S.Act8(code[:rows * cols].view(rows, cols), exp[:rows * nb].view(rows, nb))
    S.seg_act_pack(x, out)
    assert bool((code[rows * cols:] == 77).all()) and bool((exp[rows * nb:] == 77).all())
    for dt in (torch.bfloat16, torch.float32):
        v = torch.full((rows * cols + 999,), 77, dtype=dt, device="cuda")
        S.seg_act_unpack(out, x=v[:rows * cols].view(rows, cols))
        assert bool((v[rows * cols:] == 77).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,wide", [(200000, 3, 3), (150000, 33, 37), (5000, 1001, 1001), (1200, 18944, 18944), (9001, 4003, 4007)])
def test_large_tensors_equal_their_parts(rows, cols, wide, dtype):
    """Four chunks a lane, through the caches and (the last two) past them: every row as in calls
    of a few rows, which take one chunk a lane and equal the oracle above; nothing behind the
    end or between the rows is written."""
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(cols)
    base = torch.randn(rows, wide, generator=gen, device="cuda")
    base *= torch.exp(3 * torch.randn(rows, 1, generator=gen, device="cuda"))
    base = base.to(dt)
    x = base[:, wide - cols:]
    x[rows // 3] = 0
    x[rows // 2, cols - 1] = float("inf")
    nb = -(-cols // 32)
    part = (1 << 19) // (nb * (4 if dtype == "bf16" else 8))
    assert part < rows
    say(f"{rows} x {cols} of {wide} {dtype}, parts of {part}")
    code = torch.full((rows * cols + 4096,), 77, dtype=torch.int8, device="cuda")
    exp = torch.full((rows * nb + 4096,), 77, dtype=torch.uint8, device="cuda")
    a = S.Act8(code[:rows * cols].view(rows, cols), exp[:rows * nb].view(rows, nb))
    S.seg_act_pack(x, a)
    assert bool((code[rows * cols:] == 77).all()) and bool((exp[rows * nb:] == 77).all())
    out = torch.full((rows + 1, wide), 7.0, dtype=dt, device="cuda")
    S.seg_act_unpack(a, x=out[:rows, wide - cols:])
    assert bool((out[rows:] == 7).all()) and bool((out[:, :wide - cols] == 7).all())
    for r in range(0, rows, part):
        s = slice(r, min(r + part, rows))
        p = S.seg_act_pack(x[s])
        assert torch.equal(a.code[s], p.code) and torch.equal(a.exp[s], p.exp), s
        v, w = out[s, wide - cols:], S.seg_act_unpack(p, dt)
        assert torch.equal(v.isnan(), w.isnan()) and torch.equal(v.nan_to_num(), w.nan_to_num()), s
    assert bool(a.exp[rows // 2, -1] == 255) and not a.code[rows // 3].any()
