"""8-bit floating point with blocks of 128, and its product, on the GPU.

Packing: codes, exponent bytes and values equal the float64 oracle's exactly (scaling
by a power of two rounds nothing, so the one rounding is to the nearest code).

Product, of given codes against their values in float64: scales are exact.  The matrix
instruction drops of each product what is below 2^-13 of the largest of its group of 16,
so a group is off by at most 16 2^-13 max|a| max|b| = 2^-9 max|a| max|b| of the group;
the groups' sums, and the parts of K, add up in fp32, off by at most (K / 16 + 20) 2^-24
sum|a b|; a bf16 output rounds once more, 2^-8.  Over a whole tensor of normal values the
dropped parts are independent: each at most 2^-13 of its group's largest product, about
3 of the products' size, so sqrt(1/3) 3 2^-13 < 2^-12 of the result (relative
Frobenius norm)."""
import ctypes

import numpy as np
import pytest

from oracle import fp8 as OF
from paper_2607_11185_amd import _lib
from paper_2607_11185_amd import seg as S
from tests.gpu_helpers import rel, say

pytestmark = pytest.mark.gpu

BF, F32 = "bf16", "f32"


def _dt(name):
    import torch
    return {BF: torch.bfloat16, F32: torch.float32}[name]


def _same(got, want, what):
    got = got.cpu().numpy() if hasattr(got, "cpu") else got
    bad = np.argwhere(~((got == want) | (np.isnan(got) & np.isnan(want))) if got.dtype.kind == "f" else got != want)
    if got.shape != want.shape or len(bad):
        at = tuple(bad[0])
        raise AssertionError(f"{what}: {len(bad)} differ, first at {at}: {got[at]}, not {want[at]}")


def _check(x, block_rows):
    import torch
    got = S.seg_fp8_pack(x, block_rows)
    code, exp = OF.pack(x.double().cpu().numpy(), block_rows)
    _same(got.exp, exp, "exponents")
    c = got.code.cpu().numpy()
    c = np.where((c & 127) == 127, 127, c)                 # either sign of NaN
    _same(np.where((c & 127) == 0, 0, c), np.where((code & 127) == 0, 0, code), "codes")
    want = OF.unpack(code, exp, x.shape[1], block_rows)
    _same(S.seg_fp8_unpack(got, torch.float32).double(), want, "values in fp32")
    as_bf = torch.from_numpy(want).float().bfloat16().double().numpy()   # exact but for subnormal numbers
    _same(S.seg_fp8_unpack(got).double(), as_bf, "values in bf16")
    return got


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (3, 127), (2, 128), (5, 129), (17, 100), (16, 264), (33, 1001), (127, 640),
                                       (128, 384), (129, 96), (301, 3584), (1000, 40), (2, 18944), (4099, 24), (1100, 2049)])
def test_codes_and_values(rows, cols, block_rows, dtype):
    import torch
    say(f"{rows} x {cols} blocks of {block_rows} {dtype}")
    gen = torch.Generator(device="cuda").manual_seed(rows * 7 + cols)
    x = torch.randn(rows, cols, generator=gen, device="cuda")
    x *= torch.exp(4 * torch.randn(rows, 1, generator=gen, device="cuda"))      # rows of any size
    x[torch.rand(rows, cols, generator=gen, device="cuda") < 0.1] = 0
    if rows > 3:
        x[2] = 0
    _check(x.to(_dt(dtype)), block_rows)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("cols,wide,at", [(256, 288, 16), (256, 261, 4), (200, 231, 3), (128, 129, 1)])
def test_parts_of_wider_rows(cols, wide, at, block_rows, dtype):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(cols)
    base = torch.randn(137, wide, generator=gen, device="cuda").to(_dt(dtype))
    got = _check(base[:, at:at + cols], block_rows)
    out = torch.full_like(base, 7.0)
    S.seg_fp8_unpack(got, x=out[:, at:at + cols])
    assert torch.equal(out[:, at:at + cols], S.seg_fp8_unpack(got, out.dtype))
    assert bool((out[:, :at] == 7).all()) and bool((out[:, at + cols:] == 7).all())


@pytest.mark.parametrize("block_rows", [1, 128])
def test_numbers_at_the_edges(block_rows):
    """Largest and smallest numbers, ties between codes, infinities and NaN."""
    import torch
    t = OF.numbers()
    ties = np.concatenate([(t[1:] + t[:-1]) / 2, -(t[1:] + t[:-1]) / 2, np.nextafter(((t[1:] + t[:-1]) / 2).astype(np.float32), np.float32(9e9))])
    x = torch.zeros(160, 384, dtype=torch.float32, device="cuda")
    x[0, :128] = torch.from_numpy(ties[:128]).float()
    x[0, 0] = 448.0
    x[130, 128:256] = torch.from_numpy(ties[126:254]).float()
    x[130, 129] = -448.0
    x[131, :126] = torch.from_numpy(ties[252:378]).float()
    x[1, 0], x[1, 1] = float("inf"), 3.0
    x[2, 5], x[2, 6], x[2, 200] = float("nan"), -float("inf"), 2.5
    x[3, 256:] = torch.logspace(-45, 38, 128, device="cuda")
    x[140, 256:] = -3.4028234663852886e38
    x[141, 256:] = torch.linspace(3.0e38, 3.4e38, 128, device="cuda")
    x[142, :] = 1e-45
    x[143, 128:256] = torch.logspace(-45, -37, 128, device="cuda")
    _check(x, block_rows)


def test_arrays_are_written_whole():
    """Zero codes behind the columns, zero bytes behind the last block of rows, whatever lay there."""
    import torch
    for block_rows in (1, 128):
        x = torch.randn(37, 133, device="cuda")
        out = S.Fp8.empty(37, 133, block_rows, "cuda")
        out.code.fill_(0x55)
        out.exp.fill_(0x55)
        S.seg_fp8_pack(x, block_rows, out)
        assert bool((out.code[:, 133:] == 0).all())
        n = -(-37 // block_rows)
        assert bool((out.exp[:, n:] == 0).all()) and bool((out.exp[:, :n] > 0).all())


def test_packing_of_no_rows():
    import torch
    a = S.seg_fp8_pack(torch.empty(0, 5, device="cuda"))
    assert S.seg_fp8_unpack(a).shape == (0, 5)
    b = S.seg_fp8_pack(torch.randn(3, 5, device="cuda"))
    assert S.seg_fp8_gemm(a, b).shape == (0, 3)


# ---------------------------------------------------------------- the product

def _operands(rows, outs, cols, ba=1, bb=128, seed=0):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed * 1000 + rows + outs)
    x = torch.randn(rows, cols, generator=gen, device="cuda")
    w = torch.randn(outs, cols, generator=gen, device="cuda")
    # blocks of different sizes along both sides
    x *= torch.exp2(torch.randint(-6, 6, (rows, -(-cols // 128)), generator=gen, device="cuda").float()).repeat_interleave(128, 1)[:, :cols]
    w *= torch.exp2(torch.randint(-6, 6, (outs, -(-cols // 128)), generator=gen, device="cuda").float()).repeat_interleave(128, 1)[:, :cols]
    return S.seg_fp8_pack(x, ba), S.seg_fp8_pack(w, bb)


def _values(a):
    return OF.unpack(a.code.cpu().numpy(), a.exp.cpu().numpy(), a.cols, a.block_rows)


def _groups(v):
    pad = np.pad(np.abs(v), ((0, 0), (0, -v.shape[1] % 16)))
    return pad.reshape(len(v), -1, 16).max(2)


def _product(a, b):
    """Values of a b^T in float64, and how far fp32 results may be off."""
    va, vb = _values(a), _values(b)
    tol = 2.0 ** -9 * (_groups(va) @ _groups(vb).T)
    tol += (a.cols / 16 + 20) * 2.0 ** -24 * (np.abs(va) @ np.abs(vb).T)
    return va @ vb.T, tol + 1e-40


def _within(got, ref, tol, what):
    got = got.double().cpu().numpy()
    over = np.abs(got - ref) - tol
    assert got.shape == ref.shape and float(over.max()) <= 0, (what, float(over.max()), int((over > 0).sum()))


SHAPES = [(1, 1, 1), (1, 16, 128), (1, 300, 1000), (3, 33, 129), (16, 64, 256), (17, 100, 2040), (32, 2048, 640), (33, 31, 1300),
          (64, 130, 4096), (65, 7, 100), (70, 257, 513), (130, 520, 1111), (257, 256, 2048), (300, 1032, 128), (777, 5001, 2040),
          (128, 640, 9001), (2, 40, 16384),
          # each kernel for few rows, and each kind of tile
          (5, 4200, 2200), (9, 48, 2304), (20, 4200, 300), (25, 100, 1500), (40, 100, 1500), (50, 4200, 700), (47, 16500, 300),
          (300, 12000, 128), (400, 19000, 128), (65, 12000, 4096), (130, 5000, 16384), (130, 19000, 128), (65, 5504, 16384),
          (700, 5504, 128), (1400, 1300, 16384), (257, 200, 17000), (40, 9000, 4000), (33, 3000, 12000)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("ba,bb", [(1, 128), (1, 1), (128, 1), (128, 128)])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_product(shape, ba, bb, dtype):
    say(shape, ba, bb, dtype)
    a, b = _operands(*shape, ba, bb)
    got = S.seg_fp8_gemm(a, b, _dt(dtype))
    ref, tol = _product(a, b)
    _within(got, ref, tol + (2.0 ** -8 * (np.abs(ref) + tol) if dtype == BF else 0), "y")


def test_every_way_of_cutting():
    """The shapes take each kernel, whole and in parts of K."""
    L = _lib.lib()
    f = L.seg_fp8_gemm_choice
    f.restype, f.argtypes = None, [ctypes.c_int32] * 3 + [ctypes.c_void_p]
    got = set()
    for s in SHAPES:
        out = (ctypes.c_int32 * 3)()
        f(*s, out)
        got.add((out[0], out[1], min(out[2], 2)))
        assert (L.seg_fp8_gemm_workspace_bytes(*s) > 0) == (out[2] > 1)
    # 16-row blocks of a, of b, waves
    assert got >= {(1, 1, -16), (1, 1, -8), (2, 1, -8), (2, 2, -4), (4, 1, -8), (4, 2, -8), (4, 4, -4)}, got
    # 256 x 256 tiles, 128 x 256, 128 x 128 two and one to a CU, whole and in parts of K
    assert got >= {(v, 0, p) for v in range(4) for p in (1, 2)}, got


@pytest.mark.parametrize("shape", [(40, 512, 4096), (513, 1024, 4096), (2, 256, 8192)], ids=lambda s: "x".join(map(str, s)))
def test_rate_of_error(shape):
    """Over a whole tensor of normal values."""
    import torch
    rows, outs, cols = shape
    gen = torch.Generator(device="cuda").manual_seed(5)
    a = S.seg_fp8_pack(torch.randn(rows, cols, generator=gen, device="cuda"))
    b = S.seg_fp8_pack(torch.randn(outs, cols, generator=gen, device="cuda"), 128)
    ref = _values(a) @ _values(b).T
    e = rel(S.seg_fp8_gemm(a, b, torch.float32).cpu().numpy(), ref)
    say(shape, e)
    assert e < 2.0 ** -12


@pytest.mark.parametrize("rows", [5, 30, 64, 300])
def test_not_a_number_stays_in_its_row_and_column(rows):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, 700, generator=gen, device="cuda")
    w = torch.randn(270, 700, generator=gen, device="cuda")
    clean = S.seg_fp8_gemm(S.seg_fp8_pack(x), S.seg_fp8_pack(w, 128))
    x[3, 650], w[131, 2], w[200, 699] = float("inf"), float("nan"), -float("inf")
    got = S.seg_fp8_gemm(S.seg_fp8_pack(x), S.seg_fp8_pack(w, 128))
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[3], bad[:, 131], bad[:, 200] = True, True, True
    assert torch.equal(got.isnan(), bad)
    # (a block's scale may have changed with its largest value: columns of other blocks are the same)
    assert torch.equal(got[4:, :128], clean[4:, :128])


@pytest.mark.parametrize("rows", [2, 100])
def test_blocks_of_very_different_size(rows):
    """Scales from the smallest to the largest: each block by itself, and sums that leave fp32."""
    import torch
    x = torch.zeros(rows, 256, device="cuda")
    w = torch.zeros(40, 256, device="cuda")
    x[:, :128], w[:, :128] = 2.0 ** -120, 2.0 ** 115
    x[1, 128:], w[7, 128:] = 2.0 ** 100, 2.0 ** 100
    got = S.seg_fp8_gemm(S.seg_fp8_pack(x), S.seg_fp8_pack(w), torch.float32)
    want = torch.full((rows, 40), 128 * 2.0 ** -5, device="cuda")
    want[1, 7] = float("inf")
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("shape", [(7, 45, 300), (100, 301, 300), (80, 24, 8192)], ids=lambda s: "x".join(map(str, s)))
def test_outputs_in_wider_rows(shape, dtype):
    """Into the middle of rows at any distance; nothing else is written."""
    import torch
    rows, outs, cols = shape
    a, b = _operands(*shape)
    wide = torch.full((rows + 2, outs + 9), 7.0, dtype=_dt(dtype), device="cuda")
    n = _lib.lib().seg_fp8_gemm_workspace_bytes(rows, outs, cols)
    ws = torch.full((n + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    S.seg_fp8_gemm(a, b, y=wide[1:-1, 3:3 + outs], ws=ws[:n] if n else None)
    assert torch.equal(wide[1:-1, 3:3 + outs], S.seg_fp8_gemm(a, b, wide.dtype))
    wide[1:-1, 3:3 + outs] = 7.0
    assert bool((wide == 7).all()) and bool((ws[n:] == 0x5A).all())


@pytest.mark.parametrize("shape", [(4, 96, 1000), (90, 40, 8192), (600, 512, 1024)], ids=lambda s: "x".join(map(str, s)))
def test_graph_streams_and_repeats(shape):
    """Captured and replayed with new inputs between the replays, and on another stream: the same bits."""
    import torch
    a, b = _operands(*shape)
    ws = S.fp8_gemm_workspace(*shape, "cuda")
    x = S.seg_fp8_unpack(a, torch.float32)
    y = torch.empty(shape[0], shape[1], dtype=torch.bfloat16, device="cuda")
    S.seg_fp8_gemm(S.seg_fp8_pack(x, 1, a), b, y=y, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.seg_fp8_pack(x, 1, a)
        S.seg_fp8_gemm(a, b, y=y, ws=ws)
    for i in range(3):
        x.copy_(torch.randn_like(x) * (i + 1))
        graph.replay()
        got = y.clone()
        want = S.seg_fp8_gemm(S.seg_fp8_pack(x), b)
        assert torch.equal(got, want), i
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = S.seg_fp8_gemm(S.seg_fp8_pack(x), b)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(other, want)


def test_large_outputs_past_32_bits():
    """Offsets of y past 2^31 elements."""
    import torch
    rows, outs, cols = 40000, 57344, 32
    a, b = _operands(rows, outs, cols)
    y = S.seg_fp8_gemm(a, b)
    at = torch.tensor([0, 1, 37449, 37450, 39998, 39999], device="cuda")
    part = S.Fp8(a.code[at].contiguous(), torch.nn.functional.pad(a.exp[:, at], (0, 10)).contiguous(), cols, 1)
    ref, tol = _product(part, b)
    _within(y[at], ref, tol + 2.0 ** -8 * (np.abs(ref) + tol), "rows")


@pytest.mark.parametrize("block_rows", [1, 128])
def test_packing_past_32_bits(block_rows):
    """Rows behind 2^32 bytes of x and 2^31 codes."""
    import torch
    rows, cols = 600001, 4100
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(130, cols, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    at = rows - 130 if block_rows == 1 else (rows - 1) // 128 * 128 - 65
    x[at:at + 130] = tail[:rows - at]
    x[7, 4099] = 3.0
    a = S.seg_fp8_pack(x, block_rows)
    first = at // 128 * 128
    want = S.seg_fp8_unpack(S.seg_fp8_pack(x[first:].contiguous(), block_rows))
    got = S.seg_fp8_unpack(a)
    assert torch.equal(got[first:], want) and bool(want[at - first:].any())
    assert float(got[7, 4099]) == 3.0 and int(got[:first].count_nonzero()) == 1


@pytest.mark.parametrize("rows", [3, 200])
def test_the_byte_that_stands_for_nan(rows):
    """255 in an exponent array reads as NaN, and makes NaN of its block's rows and columns."""
    import torch
    a, b = _operands(rows, 150, 300)
    want = S.seg_fp8_gemm(a, b)
    a.exp[1, 2] = 255
    b.exp[2, 1] = 255                                      # columns 128 to 149 of y
    got = S.seg_fp8_gemm(a, b)
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[2], bad[:, 128:] = True, True
    assert torch.equal(got.isnan(), bad) and torch.equal(got[~bad], want[~bad])
    v = S.seg_fp8_unpack(a)
    assert bool(v[2, 128:256].isnan().all()) and not bool(v[2, :128].isnan().any()) and not bool(v[0].isnan().any())


@pytest.mark.parametrize("rows,outs,cols", [(1 << 20, 5, 16), (3, 1 << 20, 24), (66, (1 << 20) - 3, 16), (70, 9, 1 << 20)])
def test_largest_sizes(rows, outs, cols):
    """Against a product of the values in fp32, exact but for its order: codes of whole numbers."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(cols)
    # whole numbers up to 4: products and sums of them are exact everywhere
    x = torch.randint(-4, 5, (rows, cols), generator=gen, device="cuda").float()
    w = torch.randint(-4, 5, (outs, cols), generator=gen, device="cuda").float()
    got = S.seg_fp8_gemm(S.seg_fp8_pack(x), S.seg_fp8_pack(w, 128), torch.float32)
    assert torch.equal(got, x @ w.t())


@pytest.mark.parametrize("rows,cols,block_rows", [(1 << 27, 1, 1), ((1 << 28) + 5, 1, 128)])
def test_largest_launches(rows, cols, block_rows):
    """Of 2^23 thread blocks, and more rows in blocks of 128 than of one: parts packed alone."""
    import torch
    x = torch.randn(rows, cols, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda", dtype=torch.bfloat16)
    a = S.seg_fp8_pack(x, block_rows)
    for at in (0, rows // 256 * 128, rows // 128 * 128 - 4096):
        to = min(rows, at + 100000)
        part = S.seg_fp8_pack(x[at:to], block_rows)
        n, first = -(-(to - at) // block_rows), at // block_rows
        assert torch.equal(a.code[at:to], part.code) and torch.equal(a.exp[:, first:first + n], part.exp[:, :n])
    if block_rows == 1:
        got = S.seg_fp8_unpack(a)
        for at in (0, rows // 256 * 128, rows - 100000):
            assert torch.equal(got[at:at + 100000], S.seg_fp8_unpack(S.seg_fp8_pack(x[at:at + 100000])))


def test_widest_row():
    """2^30 columns: a block of 128 rows that holds one is the block of that row."""
    import torch
    x = torch.randn(1, 1 << 30, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda", dtype=torch.bfloat16)
    x[0, -128:] *= 1000
    a, b = S.seg_fp8_pack(x), S.seg_fp8_pack(x, 128)
    assert torch.equal(a.code, b.code) and torch.equal(a.exp, b.exp)
    part = S.seg_fp8_pack(x[:, -1280:], 128)
    assert torch.equal(part.code, b.code[:, -1280:]) and torch.equal(part.exp, b.exp[-10:])


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,cols,dtype", [(9000, 4099, BF), (5133, 4099, F32)])
def test_tensors_past_the_caches(rows, cols, dtype, block_rows):
    """More than 96 MB in and out, read and written past the caches: as their parts alone."""
    import torch
    x = torch.randn(rows, cols, generator=torch.Generator(device="cuda").manual_seed(rows), device="cuda").to(_dt(dtype))
    a = S.seg_fp8_pack(x, block_rows)
    got = S.seg_fp8_unpack(a, x.dtype)
    for at in range(0, rows, 1024):
        part = S.seg_fp8_pack(x[at:at + 1024], block_rows)
        n = -(-part.shape[0] // block_rows)
        assert torch.equal(a.code[at:at + 1024], part.code)
        assert torch.equal(a.exp[:, at // block_rows:at // block_rows + n], part.exp[:, :n])
        assert torch.equal(got[at:at + 1024], S.seg_fp8_unpack(part, x.dtype))
