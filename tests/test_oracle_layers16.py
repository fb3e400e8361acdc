"""The oracle of the 16-bit layers against closed forms: linear attention as one masked product and as blocks joined by
their states, the activations at known points."""
import math

import numpy as np
import pytest

import oracle as O


def test_linear_attention_equals_the_masked_product():
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(2, 19, 2, 5)), rng.normal(size=(2, 19, 2, 5)), rng.normal(size=(2, 19, 4, 3))
    g = -rng.random((2, 19, 4))
    out, S, _, _ = O.linattn(q, k, v, g, scale=0.5)
    G = np.cumsum(g, axis=1)
    for b in range(2):
        for h in range(4):
            D = np.tril(np.exp(np.minimum(G[b, :, None, h] - G[b, None, :, h], 0.0)))
            want = 0.5 * (q[b, :, h // 2] @ k[b, :, h // 2].T * D) @ v[b, :, h]
            assert np.allclose(out[b, :, h], want, rtol=0, atol=1e-12)
            assert np.allclose(S[b, h], (k[b, :, h // 2] * np.exp(G[b, -1:, h] - G[b, :, h])[:, None]).T @ v[b, :, h], rtol=0, atol=1e-12)


def test_linear_attention_continues_from_its_state_and_stops_at_the_lengths():
    rng = np.random.default_rng(1)
    q, k, v = (rng.normal(size=(3, 12, 1, 4)) for _ in range(3))
    g = -rng.random((3, 12, 1))
    whole, S, size, _ = O.linattn(q, k, v, g)
    a, Sa, _, _ = O.linattn(q[:, :7], k[:, :7], v[:, :7], g[:, :7])
    b, Sb, _, _ = O.linattn(q[:, 7:], k[:, 7:], v[:, 7:], g[:, 7:], state=Sa)
    assert np.allclose(whole, np.concatenate([a, b], 1), rtol=0, atol=1e-13) and np.allclose(S, Sb, rtol=0, atol=1e-13)
    assert (np.abs(whole) <= size + 1e-13).all()
    part, Sp, _, _ = O.linattn(q, k, v, g, state=S, lens=[7, 0, 12])
    assert np.array_equal(Sp[1], S[1]) and np.isnan(part[0, 7:]).all() and np.isnan(part[1]).all()
    # a decay of -infinity starts anew, a positive one counts as none
    cut = g.copy()
    cut[:, 7] = -np.inf
    again, _, _, _ = O.linattn(q, k, v, cut)
    fresh, _, _, _ = O.linattn(q[:, 7:], k[:, 7:], v[:, 7:], g[:, 7:])
    assert np.allclose(again[:, 7:], fresh, rtol=0, atol=1e-13)
    assert np.array_equal(O.linattn(q, k, v, np.ones(1))[0], O.linattn(q, k, v)[0])


@pytest.mark.parametrize("act, at, want", [("none", -2.5, -2.5), ("relu", -1.0, 0.0), ("relu", 3.0, 3.0), ("silu", 0.0, 0.0),
                                           ("silu", 1.0, 1 / (1 + math.exp(-1))), ("sigmoid", 0.0, 0.5),
                                           ("gelu", 1.0, 0.8413447460685429), ("gelu", -1.0, -0.15865525393145707),
                                           ("gelu_tanh", 1.0, 0.8411919906082768)])
def test_activations(act, at, want):
    assert O.activate(np.array([at]), act)[0] == pytest.approx(want, rel=1e-12)


def test_linear_adds_bias_before_and_residual_after_the_activation():
    x, W = np.array([[1.0, 2.0]]), np.array([[3.0, -4.0], [0.5, 1.0]])
    out, size = O.linear(x, W, bias=np.array([1.0, -3.0]), residual=np.array([[10.0, 20.0]]), act="relu")
    assert np.array_equal(out, [[10.0, 20.0]]) and np.array_equal(size, [[12.0, 5.5]])
