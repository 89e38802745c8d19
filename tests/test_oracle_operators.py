"""Pins of the oracle of the operators around the linear layers: gradients against central differences,
closed forms, and identities."""
import numpy as np
import pytest

from oracle import operators as op


def differences(f, x, dy, h=1e-5):
    """Gradient of sum(f(x) * dy) by central differences (error ~ h^2: 1e-9 of smooth functions of order 1)."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        g[i] = ((f(a) - f(b)) * dy).sum() / (2 * h)
    return g


@pytest.mark.parametrize("starts", [[0, 5], [0, 1, 1, 4, 6]])
def test_attention_gradients_against_differences(starts):
    rs = np.random.default_rng(0)
    T, hq, hkv, d = 7, 4, 2, 3
    q, k, v, do = (rs.standard_normal((T, h, d)) for h in (hq, hkv, hkv, hq))
    dq, dk, dv = op.attention_backward(starts, q, k, v, do, 0.7)
    f = lambda q, k, v: op.attention_forward(starts, q, k, v, 0.7)[0]
    for got, want in ((dq, differences(lambda x: f(x, k, v), q, do)), (dk, differences(lambda x: f(q, x, v), k, do)),
                      (dv, differences(lambda x: f(q, k, x), v, do))):
        assert np.abs(got - want).max() < 1e-7


def test_attention_closed_forms():
    rs = np.random.default_rng(1)
    q, k, v = rs.standard_normal((6, 2, 4)), rs.standard_normal((6, 1, 4)), rs.standard_normal((6, 1, 4))
    o, lse = op.attention_forward([0, 3, 5], q, k, v, 0.5)
    assert np.allclose(o[0], v[0]) and np.allclose(o[3], v[3])                    # a first token sees itself alone
    assert np.allclose(lse[0], 0.5 * (q[0] @ k[0, 0]))
    assert not o[5].any() and np.all(lse[5] == -np.inf)                           # a token of no sequence
    o, lse = op.attention_forward([0, 6], np.zeros_like(q), k, v, 0.5)           # equal scores: means
    for i in range(6):
        assert np.allclose(o[i], v[:i + 1].mean(0)) and np.allclose(lse[i], np.log(i + 1))


@pytest.mark.parametrize("center", [False, True])
def test_norm_gradients_against_differences(center):
    rs = np.random.default_rng(2)
    x, w, b, dy = rs.standard_normal((3, 7)) + 0.5, rs.standard_normal(7), rs.standard_normal(7), rs.standard_normal((3, 7))
    dx, dw, db = op.norm_backward(x, w, dy, 1e-3, center)
    f = lambda x, w, b: op.norm_forward(x, w, b, 1e-3, center)[0]
    for got, want in ((dx, differences(lambda t: f(t, w, b), x, dy)), (dw, differences(lambda t: f(x, t, b), w, dy)),
                      (db, differences(lambda t: f(x, w, t), b, dy))):
        assert np.abs(got - want).max() < 1e-7


def test_norm_identities():
    rs = np.random.default_rng(3)
    x = rs.standard_normal((4, 9))
    y, mean, _ = op.norm_forward(x, np.ones(9), None, 0.0, True)
    assert np.allclose(y.mean(1), 0) and np.allclose((y ** 2).mean(1), 1) and np.allclose(mean, x.mean(1))
    assert np.allclose(op.norm_forward(x + 7, np.ones(9), None, 0.0, True)[0], y)         # shifts do not matter
    z = op.norm_forward(x, np.ones(9), None, 0.0, False)[0]
    assert np.allclose((z ** 2).mean(1), 1) and np.allclose(op.norm_forward(5 * x, np.ones(9), None, 0.0, False)[0], z)


def test_embedding_is_a_product_with_one_hot_rows():
    rs = np.random.default_rng(4)
    ids = [3, 0, 3, -1, 5, 4, 3]
    table, dout = rs.standard_normal((5, 4)), rs.standard_normal((7, 4))
    hot = np.array([[float(i == v) for v in range(5)] for i in ids])
    assert np.allclose(op.embedding_forward(ids, table, 1.5), 1.5 * hot @ table)
    assert np.allclose(op.embedding_backward(ids, dout, 1.5, 5), 1.5 * hot.T @ dout)


def test_distill_gradient_against_differences():
    rs = np.random.default_rng(5)
    z, teacher = rs.standard_normal((4, 6)), rs.standard_normal((4, 3))
    ids = np.array([[1, 4, 2], [0, 0, 5], [3, -1, 6], [-1, 9, 6]])                # twice the same; absent ones; none
    w = np.array([1.0, 0.5, 2.0, 1.0])
    loss, dz = op.distill_loss(z, ids, teacher, w, 1.7, 0.3)
    f = lambda t: op.distill_loss(t, ids, teacher, w, 1.7, 0.3)[0]
    assert np.abs(dz - differences(f, z, np.full(4, 0.3))).max() < 1e-8
    assert loss[3] == 0 and not dz[3].any()


def test_distill_of_one_label_is_cross_entropy_and_of_itself_is_zero():
    rs = np.random.default_rng(6)
    z = rs.standard_normal((3, 5))
    loss, _ = op.distill_loss(z, [[2], [0], [4]], np.zeros((3, 1)), None, 1.0, 1.0)
    lse = np.log(np.exp(z).sum(1))
    assert np.allclose(loss, [lse[0] - z[0, 2], lse[1] - z[1, 0], lse[2] - z[2, 4]])
    loss, dz = op.distill_loss(z, np.tile(np.arange(5), (3, 1)), z + 3, None, 2.0, 1.0)   # teacher = student: no divergence
    assert np.allclose(loss, 0) and np.allclose(dz, 0)


def test_attention_where_all_scores_are_minus_infinity():
    """The first key is infinite, against all queries: the first query has nothing else, the others leave it out."""
    rs = np.random.default_rng(3)
    q, k, v = (rs.standard_normal((4, 1, 3)) for _ in range(3))
    q[..., 1] = -1 - np.abs(q[..., 1])
    k[0, 0, 1] = np.inf
    with np.errstate(invalid="ignore"):
        o, lse = op.attention_forward([0, 4], q, k, v, 0.5)
    assert lse[0, 0] == -np.inf and np.isnan(o[0]).all()
    for i in range(1, 4):
        s = 0.5 * k[1:i + 1, 0] @ q[i, 0]
        assert np.allclose(lse[i, 0], np.log(np.exp(s).sum())) and np.allclose(o[i, 0], np.exp(s) @ v[1:i + 1, 0] / np.exp(s).sum())
