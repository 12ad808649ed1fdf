"""Pins of the oracle's three-axis positions, 8-bit activations and gated
block: values worked by hand, closed forms, central differences (CPU)."""
import math

import numpy as np
import pytest

from oracle import act8 as OA8
from oracle import glu as OG
from oracle import layer as OLY
from oracle import layout as OL
from oracle import mrope as OM
from paper_2607_11185_amd import workload as WL


def test_positions_by_hand():
    # prompt of 2, a 2 x 3 screenshot, 2 tokens of text, a clip of 2 frames of 1 x 2 with time step 5, 1 token
    kind = [0, 0] + [1] * 6 + [2, 2] + [1] * 4 + [2]
    step = [0, 0] + [1] * 6 + [1, 1] + [2] * 4 + [2]
    grid = {1: (1, 2, 3, 1), 2: (2, 1, 2, 5)}
    got = OM.segment_positions(kind, step, grid.__getitem__)
    want = [[0, 0, 0], [1, 1, 1],
            [2, 2, 2], [2, 2, 3], [2, 2, 4], [2, 3, 2], [2, 3, 3], [2, 3, 4],
            [5, 5, 5], [6, 6, 6],
            [7, 7, 7], [7, 7, 8], [12, 7, 7], [12, 7, 8],
            [13, 13, 13]]
    assert got.T.tolist() == want


def test_positions_of_single_patches_are_rows():
    """Screenshots of one patch, or of single rows or columns of patches, advance
    like text on their long axis; all text: the row in the segment."""
    sp = WL.explicit_spans([4], [3], [1, 5, 5, 0], [2, 3, 1, 4], [1, 1, 1, 1])
    lay = OL.build(sp, 2, 4, 128, with_tiles=False)
    grid = np.array([[1, 1, 1, 1], [1, 5, 1, 1], [1, 1, 5, 1], [0, 0, 0, 0]])
    pos = OM.positions(lay, sp, grid, lay.packed_tokens)
    rows = OLY.segment_positions(lay.segments, lay.packed_tokens)
    assert np.array_equal(pos.max(0), rows)


def test_rotation_reduces_to_one_axis_and_is_orthogonal():
    rng = np.random.default_rng(0)
    x, y = rng.standard_normal((2, 9, 3, 32))
    p = rng.integers(0, 10000, 9)
    one = OM.rotate(x, np.stack([p, p * 0, p * 0]), (16, 0, 0), 1e4)
    assert np.allclose(one, OLY.rope(x, p, 1e4))
    pos = rng.integers(0, 10000, (3, 9))
    pos[1, 4] = -1
    z = OM.rotate(x, pos, (4, 5, 7), 1e4)
    assert np.array_equal(z[4], x[4])
    ok = np.arange(9) != 4
    assert np.allclose(np.linalg.norm(z, axis=-1), np.linalg.norm(x, axis=-1))
    back = OM.rotate(y, pos, (4, 5, 7), 1e4, inverse=True)
    assert np.isclose((z[ok] * y[ok]).sum(), (x[ok] * back[ok]).sum()) and not back[4].any()
    # one pair by hand: pair 5 is on the height axis, and 32^(-10/32) of its position
    t = pos[1, 0] * 1e4 ** (-10 / 32)
    assert np.isclose(z[0, 1, 5], x[0, 1, 5] * math.cos(t) - x[0, 1, 21] * math.sin(t))


@pytest.mark.parametrize("top,byte", [(0.0, 0), (1e-45, 0), (127.0, 127), (127.0 * (1 + 2 ** -23), 128), (126.9, 127),
                                      (63.5, 126), (64.0, 127), (1.0, 121), (2.0 ** 127, 248),
                                      (float(np.finfo(np.float32).max), 249), (math.inf, 255), (math.nan, 255)])
def test_exponent_bytes_by_hand(top, byte):
    assert OA8.exponent(top) == byte


def test_pack_values():
    x = np.array([[127.0, -3.5, 2.5, 0.4] + [0.0] * 28 + [1.0, -0.5]])
    code, exp = OA8.pack(x)
    assert exp.tolist() == [[127, 121]] and code[0, :4].tolist() == [127, -4, 2, 0] and code[0, 32:].tolist() == [64, -32]
    assert OA8.unpack(code, exp)[0, 32:].tolist() == [1.0, -0.5]
    rng = np.random.default_rng(1)
    x = rng.standard_normal((20, 75)) * np.exp(rng.standard_normal((20, 1)) * 20)
    v = OA8.unpack(*OA8.pack(x))
    for b in range(3):
        at = slice(32 * b, min(75, 32 * b + 32))
        top = np.abs(x[:, at]).max(1, keepdims=True)
        assert (np.abs(v - x)[:, at] <= top / 127).all()       # half a step, and a step is at most top / 63.5
    assert np.array_equal(OA8.unpack(*OA8.pack(v)), v)         # values are kept as they are
    x[3, 40] = math.inf
    x[4, 70] = math.nan
    v = OA8.unpack(*OA8.pack(x))
    assert np.isnan(v[3, 32:64]).all() and np.isnan(v[4, 64:]).all() and np.isfinite(v[3, :32]).all()


def test_gated_block_gradients_against_differences():
    rng = np.random.default_rng(2)
    x, wg, wu, dm = (rng.standard_normal(s) for s in ((5, 6), (4, 6), (4, 6), (5, 4)))
    m, g, u = OG.forward(x, wg, wu)
    grads = OG.backward(x, wg, wu, g, u, dm)
    for t, got in zip((x, wg, wu), grads):
        num = np.zeros_like(t)
        for i in np.ndindex(t.shape):
            old, h = t[i], 1e-5
            t[i] = old + h
            hi = (OG.forward(x, wg, wu)[0] * dm).sum()
            t[i] = old - h
            lo = (OG.forward(x, wg, wu)[0] * dm).sum()
            t[i] = old
            num[i] = (hi - lo) / (2 * h)
        # the third derivatives are of order 10 here: h^2 of them, and 1e-16 of the sum over h
        assert np.abs(num - got).max() < 1e-8 * max(1.0, np.abs(got).max()) * 10
