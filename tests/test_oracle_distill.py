"""The oracle of the distillation loss against closed forms and differences (CPU)."""
import numpy as np
import pytest

from oracle import distill as OD
from oracle import fp8 as OF
from oracle import top as OT


def _case(rows=3, hidden=8, vocab=20, k=5, seed=0, given=False):
    r = np.random.default_rng(seed)
    h, w = r.normal(size=(rows, hidden)), r.normal(size=(vocab, hidden))
    ids = np.stack([r.permutation(vocab)[:k] for _ in range(rows)]).astype(np.int32)
    logits = r.normal(size=(rows, k)) * 2
    t_lse = np.log(np.exp(0.7 * logits).sum(1)) + 0.4 if given else None
    return h, w, ids, logits, dict(logit_scale=0.9, teacher_scale=0.7, loss_scale=0.3, t_lse=t_lse,
                                   weight=r.uniform(0.5, 2, rows))


def test_whole_vocabulary_is_the_divergence():
    """All columns as entries, and the student equal to the teacher: 0, and no gradient."""
    h, w, _, _, kw = _case()
    ids = np.tile(np.arange(20, dtype=np.int32), (3, 1))
    out = OD.loss_and_grads(h, w, ids, 0.9 * (h @ w.T) / 0.7, **kw)
    assert np.abs(out["loss_tok"]).max() < 1e-12 and np.abs(out["dz"]).max() < 1e-12


def test_one_entry_is_the_negative_log_probability():
    h, w, ids, logits, kw = _case(k=1)
    out = OD.loss_and_grads(h, w, ids, logits, **kw)
    logq = out["z"] - out["lse"][:, None]
    assert np.allclose(out["loss_tok"], -kw["weight"] * logq[np.arange(3), ids[:, 0]])


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("what", ["h", "w"])
def test_gradients_against_differences(what, given):
    h, w, ids, logits, kw = _case(given=given)
    ids[0, 3], ids[1] = -1, ids[1, 0]                    # a missing entry, and the same one five times
    out = OD.loss_and_grads(h, w, ids, logits, **kw)
    x, d = (h, out["dh"]) if what == "h" else (w, out["dw"])
    for at in [(0, 0), (1, 3), (2, 7)]:
        eps, s = 1e-6, []
        for sign in (1, -1):
            y = x.copy()
            y[at] += sign * eps
            a, b = (y, w) if what == "h" else (h, y)
            s.append(OD.loss_and_grads(a, b, ids, logits, **kw)["loss_sum"])
        assert abs((s[0] - s[1]) / (2 * eps) - d[at]) < 1e-7


def test_rows_without_entries():
    h, w, ids, logits, kw = _case()
    ids[1] = -1
    logits[2] = -np.inf
    out = OD.loss_and_grads(h, w, ids, logits, **kw)
    assert out["loss_tok"][1] == out["loss_tok"][2] == 0
    assert not out["dz"][1:].any() and out["dz"][0].any()


def test_numbers_of_the_format():
    t = OF.numbers()
    assert len(t) == 127 and t[0] == 0 and t[1] == 2.0 ** -9 and t[8] == 2.0 ** -6 and t[-1] == 448.0
    assert (np.diff(t) > 0).all()
    x = np.array([[448.0, 1.0, 1.0625, 1.1875, -0.0, 2.0 ** -10, 3 * 2.0 ** -10, 1e9]])[:, :7]
    code, exp = OF.pack(x)
    assert exp[0, 0] == 127 and exp.shape == (1, 16) and code.shape == (1, 16)
    assert OF.unpack(code, exp, 7)[0].tolist() == [448.0, 1.0, 1.0, 1.25, 0.0, 0.0, 2.0 ** -8]   # ties to even
    for top, byte in ((448.0, 127), (449.0, 128), (224.0, 126), (225.0, 127), (0.0, 0), (3.4028234663852886e38, 247)):
        assert OF.pack(np.array([[top, 0.0]]))[1][0, 0] == byte
    assert np.isfinite(OF.unpack(*OF.pack(np.full((1, 3), 3.4028234663852886e38)), 3)).all()
    assert np.float32(OF.unpack(*OF.pack(np.full((1, 3), 3.4028234663852886e38)), 3)).max() < np.inf


def test_order_of_the_selection():
    z = np.array([[1.0, np.nan, 3.0, 3.0, -np.inf, np.inf, -0.0, 0.0]])
    ids, v = OT.top(z, 8)
    assert ids[0].tolist() == [1, 5, 2, 3, 0, 6, 7, 4]
    assert np.isclose(OT.lse(np.zeros((1, 7)))[0], np.log(7)) and OT.lse(np.full((1, 3), -np.inf))[0] == -np.inf
