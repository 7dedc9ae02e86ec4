"""The reference of the int8 layers and of the routing by scores against hand-worked numbers."""
import numpy as np

from oracle import int_oracle as io


def test_rows():
    q, s = io.quantize_rows(np.array([[254.0, 1.0, -1.0, 3.0, -254.0], [0, 0, 0, 0, 0], [1.0, np.nan, 0, 0, 0], [np.inf, 1, 0, 0, 0], [1e39, 1, 0, 0, 0]]))
    assert q[0].tolist() == [127, 0, 0, 2, -127] and s[0] == 2.0            # 0.5 and -0.5 to 0, 1.5 to 2
    assert not q[1:].any() and s[1] == 2.0 ** -126 and np.isnan(s[2:]).all()
    q, s = io.quantize_rows(np.array([[3.0 * 2.0 ** -126, 1.0]]), np.array([2.0 ** -130]))
    assert s[0] == 2.0 ** -126 and q[0].tolist() == [0, 0]                  # the smallest scale: values are rounded in its units
    q, s = io.quantize_rows(np.array([[2.0 ** -120, 2.0 ** -126]]))
    assert s[0] == 2.0 ** -126 and q[0].tolist() == [64, 1]


def test_weights():
    q, s = io.quantize_weights(np.array([[127.0, 0.5, -1.5, -127.0], [0, 0, 0, 0], [np.inf, 1, 1, 1]]))
    assert q[0].tolist() == [127, 0, -2, -127] and s.tolist()[:2] == [1.0, 2.0 ** -126] and np.isnan(s[2]) and not q[1:].any()


def test_activations():
    assert io.activate(np.array([-1.0, 2.0]), "relu").tolist() == [0.0, 2.0]
    assert np.allclose(io.activate(np.array([1.0, -1.0]), "silu"), [0.7310585786300049, -0.2689414213699951], rtol=1e-15)
    assert np.allclose(io.activate(np.array([1.0, -1.0]), "gelu"), [0.8413447460685429, -0.15865525393145707], rtol=1e-15)


def test_product():
    z, size = io.product(np.array([[1, -2]]), [0.5], np.array([[3, 4], [-128, 127]]), [2.0, 1.0], [1.0, 0.0])
    assert z.tolist() == [[-4.0, -191.0]] and size.tolist() == [[5.0, 191.0]]


def test_route():
    l = np.log(np.array([[1.0, 2.0, 3.0, 4.0]]))
    idx, w = io.route(l, 2)
    assert idx.tolist() == [[3, 2]] and np.allclose(w, [[0.4, 0.3]])
    idx, w = io.route(l, 2, renormalize=True, scale=7.0)
    assert np.allclose(w, [[4.0, 3.0]])
    idx, w = io.route(l, 2, score="sigmoid")                               # p / (1 + p): 1/2, 2/3, 3/4, 4/5
    assert idx.tolist() == [[3, 2]] and np.allclose(w, [[0.8, 0.75]])
    idx, w = io.route(l, 2, score="sigmoid", balance=[0.5, 0, 0, 0])
    assert idx.tolist() == [[0, 3]] and np.allclose(w, [[0.5, 0.8]])       # the bias chooses and does not weigh
    # groups {0, 1} and {2, 3}: the largest is in the second, the larger pair too; with the bias on the first
    assert io.route(l, 2, groups=2, kept=1)[0].tolist() == [[3, 2]]
    assert io.route(l, 2, groups=2, kept=1, top=2, balance=[0.3, 0.3, 0, 0])[0].tolist() == [[1, 0]]
    m = np.log(np.array([[5.0, 0.1, 3.0, 4.0]]))                           # largest expert alone against the larger pair
    assert io.route(m, 1, groups=2, kept=1)[0].tolist() == [[0]] and io.route(m, 1, groups=2, kept=1, top=2)[0].tolist() == [[3]]
    # ties, masked experts, tokens without any
    assert io.route(np.zeros((1, 4)), 3)[0].tolist() == [[0, 1, 2]]
    idx, w = io.route(np.array([[-np.inf, 0.0, -np.inf, -np.inf]]), 3, renormalize=True)
    assert idx.tolist() == [[1, 0, 2]] and w.tolist() == [[1.0, 0.0, 0.0]]
    idx, w = io.route(np.full((1, 4), -np.inf), 2, renormalize=True)
    assert idx.tolist() == [[0, 1]] and w.tolist() == [[0.0, 0.0]]
    idx, w = io.route(np.array([[np.nan, 0.0, 1.0, 2.0]]), 2)
    assert idx.tolist() == [[3, 2]] and np.isnan(w).all()
