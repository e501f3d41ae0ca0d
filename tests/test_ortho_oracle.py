"""CPU pins of the oracle's Newton-Schulz iteration and Muon step, and the host checks of
their entry points."""
import ctypes

import numpy as np
import pytest

import __graft_entry__ as G
import oracle as O
import paper_2609_34325_gb300 as P


def _quintic(s, steps):
    a, b, c = 3.4445, -4.7750, 2.0315
    for _ in range(steps):
        s = a * s + b * s ** 3 + c * s ** 5
    return s


@pytest.mark.parametrize("shape", [(5, 9), (9, 5), (6, 6), (1, 7), (7, 1), (1, 1)])
@pytest.mark.parametrize("steps", [1, 3, 5])
def test_iteration_acts_on_the_singular_values(shape, steps):
    # odd powers of X keep its singular vectors and map its singular values one by one
    u = np.random.default_rng(1).standard_normal(shape) * 37
    left, s, right = np.linalg.svd(u, full_matrices=False)
    want = left @ np.diag(_quintic(s / np.sqrt((s * s).sum()), steps)) @ right
    assert np.allclose(O.newton_schulz(u, steps), want, atol=1e-12)


def test_singular_values_end_near_one():
    s = np.linspace(0.01, 1, 400)
    out = _quintic(s, 5)
    assert out.min() > 0.65 and out.max() < 1.21
    # the bound that the fp16 products rely on: no value ever leaves [0, 1.21]
    x = np.linspace(0, 1.21, 2000)
    assert _quintic(x, 1).min() >= 0 and _quintic(x, 1).max() < 1.21


def test_scale_of_the_update_does_not_matter():
    u = np.random.default_rng(2).standard_normal((8, 20))
    for f in (1e-300, 1e-30, 1e30, 1e150):
        assert np.allclose(O.newton_schulz(u * f), O.newton_schulz(u), atol=1e-12)
    assert not O.newton_schulz(np.zeros((3, 4))).any()


def test_muon_step_closed_forms():
    rng = np.random.default_rng(3)
    q, _ = np.linalg.qr(rng.standard_normal((6, 6)))
    p = rng.standard_normal((6, 6))
    # an orthogonal gradient, first step: the update is the gradient's own direction
    s = _quintic(np.array([1 / np.sqrt(6)]), 5)[0]
    for nesterov in (True, False):
        w, m = O.muon_step(p, 0 * p, q * 0.1, 0.5, 0.9, nesterov, 0.2, 2.0, 5, 0.25)
        assert np.allclose(m, 0.1 * 0.25 * 0.1 * q)
        assert np.allclose(w, p * (1 - 0.1) - 0.5 * 2.0 * s * q)
    # nesterov's update looks one momentum step ahead
    g, m0 = rng.standard_normal((4, 9)), rng.standard_normal((4, 9))
    _, m = O.muon_step(np.zeros((4, 9)), m0, g, 1.0, 0.8, True, 0, 1.0)
    assert np.allclose(m, 0.8 * m0 + 0.2 * g)
    w, _ = O.muon_step(np.zeros((4, 9)), m0, g, 1.0, 0.8, True, 0, 1.0)
    assert np.allclose(w, -O.newton_schulz(0.2 * g + 0.8 * m))


@pytest.fixture(scope="module")
def lib():
    G.build()
    return P.load_library()


FAR = 1 << 40                        # between buffers


def _matrix(**more):
    a = dict(grad=FAR, param=2 * FAR, momentum=3 * FAR, copy=4 * FAR, out=5 * FAR, rows=5, cols=7,
             grad_dtype=0, param_dtype=2, scale=1.0)
    a.update(more)
    return P._MatrixC(**{k: v or 0 if isinstance(v, (int, float)) else v for k, v in a.items()})


def test_list_host_checks(lib):
    def size(**more):
        return lib.dora_matrix_list_size(ctypes.byref(_matrix(**more)), 1)

    # small matrices need no memory of their own; others three copies of X in tiles of 128 x 64, an
    # even number down and across, two of the square of the shorter side
    one = size()
    assert 0 < one < 3 * 16384 and size(rows=128, cols=2048) == one
    for r, c, tiles in ((300, 200, 3 * 2 * 6 + 2 * 2 * 4), (100, 2049, 3 * 2 * 34 + 2 * 2 * 2)):
        assert tiles * 16384 <= size(rows=r, cols=c) < (tiles + 2) * 16384
    assert size(param=0, momentum=0, copy=0) == one and size(out=0) == one and size(copy=0) == one
    for bad in (dict(rows=0), dict(cols=0), dict(rows=-1), dict(grad=0), dict(grad=257),
                dict(grad_dtype=3), dict(grad_dtype=2, grad=258), dict(momentum=0),
                dict(param=0, momentum=0), dict(param=0), dict(param_dtype=-1), dict(param=258),
                dict(momentum=258), dict(copy=257), dict(out=257), dict(scale=float("nan")),
                dict(out=FAR), dict(momentum=2 * FAR + 136), dict(copy=5 * FAR - 2),
                dict(scale=float("inf")), dict(rows=16385, cols=16385),
                dict(rows=1, cols=262145), dict(rows=262145, cols=300)):
        assert size(**bad) == 0, bad
    assert lib.dora_matrix_list_size(None, 1) == 0
    assert lib.dora_matrix_list_size(ctypes.byref(_matrix()), 0) == 0
    m, l = _matrix(), P._MatrixListC()
    prepare = lib.dora_matrix_list_prepare
    assert prepare(None, 1, 256, one, ctypes.byref(l), None) == 1
    assert prepare(ctypes.byref(m), 1, None, one, ctypes.byref(l), None) == 1
    assert prepare(ctypes.byref(m), 1, 300, one, ctypes.byref(l), None) == 1
    assert prepare(ctypes.byref(m), 1, 256, one - 1, ctypes.byref(l), None) == 1
    assert prepare(ctypes.byref(m), 1, 256, one, None, None) == 1
    # an array of two: the same gradient twice may be read, nothing may be written twice
    apart = {k: 7 * FAR + i * 256 for i, k in enumerate(("param", "momentum", "copy", "out"))}

    def both(**more):
        pair = (P._MatrixC * 2)(_matrix(), _matrix(**{**apart, **more}))
        return lib.dora_matrix_list_size(pair, 2)

    assert both() > one and both(grad=FAR + 70) > one and both(param=2 * FAR + 140) > one
    for bad in (dict(param=2 * FAR), dict(momentum=3 * FAR + 136), dict(copy=4 * FAR + 68),
                dict(out=FAR + 68), dict(grad=5 * FAR + 68), dict(grad=2 * FAR - 2)):
        assert both(**bad) == 0, bad
    assert prepare((P._MatrixC * 2)(_matrix(), _matrix()), 2, 256, 1 << 30, ctypes.byref(l),
                   None) == 1


def test_call_host_checks(lib):
    l = P._MatrixListC(data=256, chunks=1, x_tiles=2, symmetric=1, outputs=1, tiles=10,
                       diagonals=1, count=1, has_params=1, has_outs=1, large=1, parts=1)
    r = ctypes.byref(l)
    assert lib.dora_orthogonalize(None, 5, None, None) == 1
    assert lib.dora_orthogonalize(r, 0, None, None) == 1
    assert lib.dora_orthogonalize(r, 33, None, None) == 1

    def step(lst=r, lr=0.1, mu=0.9, decay=0.0, steps=5):
        return lib.dora_muon_step(lst, lr, mu, 1, decay, steps, None, None, None)

    assert step(lst=None) == 1 and step(steps=0) == 1 and step(steps=33) == 1
    assert step(lr=float("nan")) == 1 and step(lr=float("inf")) == 1
    assert step(mu=1.0) == 1 and step(mu=-0.1) == 1 and step(mu=float("nan")) == 1
    assert step(decay=-1.0) == 1 and step(decay=float("inf")) == 1
    l.has_params = l.has_outs = 0
    assert lib.dora_orthogonalize(r, 5, None, None) == 1 and step() == 1
    l.has_params = l.has_outs = 1
    l.data = None
    assert lib.dora_orthogonalize(r, 5, None, None) == 1 and step() == 1


def test_binding_rejects_what_does_not_fit(lib):
    import torch
    g = torch.zeros(3, 4)
    for bad in (dict(grads=[]), dict(grads=[g]), dict(grads=[g], params=[g]),
                dict(grads=[g], copies=[g]), dict(grads=[g], scales=[1.0, 2.0])):
        with pytest.raises((TypeError, ValueError)):
            P.MatrixList(**bad)
    with pytest.raises(TypeError):
        P.dora_orthogonalize([g])
    with pytest.raises(TypeError):
        P.dora_muon_step(None, 0.1)
