"""CPU pins of the oracle's token log-probabilities and their gradient, and the host
checks of the entry points."""
import numpy as np
import pytest
import scipy.special as sp

import __graft_entry__ as G
import oracle as O
import paper_2609_34325_gb300 as P


def _inputs(seed, rows=6, classes=13):
    rng = np.random.default_rng(seed)
    return (rng.standard_normal((rows, classes)) * 2, rng.integers(0, classes, rows),
            rng.standard_normal(rows), rng.standard_normal(rows))


@pytest.mark.parametrize("temperature", [1.0, 0.6, 1.7])
def test_forward_against_scipy_and_sorting(temperature):
    z, a, _, _ = _inputs(1)
    z[2, 5] = -np.inf
    o = O.token_logprob(z, a, temperature=temperature, top=20)
    q = sp.log_softmax(z / temperature, axis=1)
    rows = np.arange(len(a))
    assert np.allclose(o["logp"], q[rows, a], atol=1e-12)
    assert np.allclose(o["entropy"], sp.entr(np.exp(q)).sum(1), atol=1e-12)
    assert np.allclose(o["norm"][:, 0] / temperature + o["norm"][:, 1],
                       sp.logsumexp(z / temperature, axis=1), atol=1e-12)
    assert np.array_equal(o["norm"][:, 0], z.max(1))
    for r in rows:
        order = np.argsort(-z[r], kind="stable")[:12 if r == 2 else 13]
        assert np.array_equal(o["top_tokens"][r, :len(order)], order)
        assert np.allclose(o["top_logp"][r, :len(order)], q[r, order], atol=1e-12)
        assert (o["top_tokens"][r, len(order):] == -1).all()
        assert np.isneginf(o["top_logp"][r, len(order):]).all()


def test_equal_logits_and_rows_without_a_part():
    z = np.array([[1., 3., 3., 2., 3.], [0., -0., 0., -0., 0.], [9., 9., 9., 9., 9.],
                  [5., 1., 2., 8., 8.], [1., 1., 1., 1., 1.]])
    o = O.token_logprob(z, [0, 1, -1, 2, -3], legal=[5, 5, 5, 3, 0], top=3)
    assert o["top_tokens"].tolist() == [[1, 2, 4], [0, 1, 2], [-1, -1, -1], [0, 2, 1],
                                        [-1, -1, -1]]
    assert np.isclose(o["entropy"][1], np.log(5)) and not o["logp"][[2, 4]].any()
    assert not O.token_logprob_grad(z, [0, 1, -1, 2, -3], np.ones(5), legal=[5, 5, 5, 3, 0])[
        [2, 4]].any()


@pytest.mark.parametrize("temperature", [1.0, 0.7])
def test_gradient_is_the_difference(temperature):
    z, a, dl, dh = _inputs(2)
    legal = np.array([13, 13, 9, 12, 13, 10])
    a = np.minimum(a, legal - 1)

    def f(x):
        o = O.token_logprob(x, a, legal, temperature)
        return (dl * o["logp"] + dh * o["entropy"]).sum()

    grad = O.token_logprob_grad(z, a, dl, dh, legal, temperature)
    h = 1e-6
    for r in range(z.shape[0]):
        for j in range(z.shape[1]):
            e = np.zeros_like(z)
            e[r, j] = h
            assert abs((f(z + e) - f(z - e)) / (2 * h) - grad[r, j]) < 1e-7
    assert np.allclose(grad.sum(1), 0, atol=1e-12)     # a shift of the logits changes nothing


@pytest.fixture(scope="module")
def lib():
    G.build()
    return P.load_library()


def test_host_checks(lib):
    def forward(logits=16, dtype=0, rows=4, classes=8, ld=8, legal=None, tokens=16, t=1.0, top=0,
                logp=16, top_logp=None, top_tokens=None):
        return lib.dora_token_logprob(logits, dtype, rows, classes, ld, legal, tokens, t, top,
                                      logp, None, None, top_logp, top_tokens, None, None)

    assert forward(logits=None) == 1 and forward(logits=17) == 1
    assert forward(logits=18, dtype=2) == 1               # fp32 at 2 bytes
    assert forward(dtype=3) == 1 and forward(dtype=-1) == 1
    assert forward(rows=-1) == 1 and forward(rows=(1 << 30) + 1) == 1
    assert forward(classes=0) == 1 and forward(ld=7) == 1
    assert forward(tokens=None) == 1 and forward(logp=None) == 1
    for t in (0.0, -1.0, float("inf"), float("nan"), 1e-39, 9e-19, 1.1e18):
        assert forward(t=t) == 1
    assert forward(top=33, top_logp=16, top_tokens=16) == 1 and forward(top=-1) == 1
    assert forward(top=2, top_logp=16) == 1 and forward(top=2, top_tokens=16) == 1

    def grad(logits=16, dtype=0, rows=4, ld=8, tokens=16, t=1.0, norm=16, entropy=None, dlogp=16,
             dentropy=None, out=16):
        return lib.dora_token_logprob_grad(logits, dtype, rows, 8, ld, None, tokens, t, norm,
                                           entropy, dlogp, dentropy, out, None, None)

    assert grad(norm=None) == 1 and grad(norm=12) == 1 and grad(out=None) == 1
    assert grad(out=17) == 1 and grad(tokens=None) == 1
    assert grad(dlogp=None) == 1 and grad(dentropy=16) == 1
    assert grad(t=0.0) == 1 and grad(ld=4) == 1


def test_binding_rejects_what_does_not_fit(lib):
    import torch
    z = torch.zeros(3, 4)
    with pytest.raises(TypeError):
        P.dora_token_logprob(z, z[0].int(), z[0])
    with pytest.raises(TypeError):
        P.dora_token_logprob_grad(z, z[0].int(), z, z)
