"""CPU pins of the oracle's policy update: gradients against differences,
closed forms of the clipping and KL terms, and the host checks of the entry
points."""
import ctypes

import numpy as np
import pytest

import __graft_entry__ as G
import oracle as O
import paper_2609_34325_gb300 as P


def _inputs(seed, rows=7, classes=11):
    rng = np.random.default_rng(seed)
    z = rng.standard_normal((rows, classes)) * 2
    a = rng.integers(0, classes, rows)
    lp = np.array([O.log_softmax(z[r])[a[r]] for r in range(rows)])
    # ratios well away from the clipping bounds, on both sides of them
    old = lp - np.where(np.arange(rows) % 3 == 0, 0.5, np.where(np.arange(rows) % 3 == 1, -0.5,
                                                              0.05))
    return z, a, old, rng.standard_normal(rows), lp + 0.3 * rng.standard_normal(rows), \
        rng.random(rows) + 0.1


@pytest.mark.parametrize("kl,ent", [(0.0, 0.0), (0.1, 0.0), (0.0, 0.05), (0.2, 0.03)])
def test_policy_gradient_is_the_loss_difference(kl, ent):
    z, a, old, adv, ref, w = _inputs(1)
    f = lambda x: O.policy_loss(x, a, old, adv, ref, w, kl_coef=kl,  # noqa: E731
                                entropy_coef=ent)["row_loss"].sum()
    grad = O.policy_loss(z, a, old, adv, ref, w, kl_coef=kl, entropy_coef=ent)["grad"]
    h = 1e-6
    for r in range(z.shape[0]):
        for j in range(z.shape[1]):
            e = np.zeros_like(z)
            e[r, j] = h
            assert abs((f(z + e) - f(z - e)) / (2 * h) - grad[r, j]) < 1e-7


def test_policy_loss_closed_forms():
    # on the policy that acted: ratio 1, loss -A, gradient -A (1(j = a) - p_j)
    z, a, _, adv, _, w = _inputs(2)
    lp = np.array([O.log_softmax(z[r])[a[r]] for r in range(len(a))])
    o = O.policy_loss(z, a, lp, adv, lp, w, kl_coef=0.7)
    assert np.allclose(o["row_loss"], -w * adv, atol=1e-12)
    p = np.exp(np.array([O.log_softmax(r) for r in z]))
    onehot = np.eye(z.shape[1])[a]
    assert np.allclose(o["grad"], (-w * adv)[:, None] * (onehot - p), atol=1e-12)
    assert o["totals"][4] == 0 and abs(o["totals"][2]) < 1e-12
    # gradients over a row add up to nothing: a shift of the logits changes nothing
    o = O.policy_loss(z, a, lp + 0.1, adv, lp - 0.2, w, kl_coef=0.7, entropy_coef=0.3)
    assert np.allclose(o["grad"].sum(1), 0, atol=1e-12)
    # clipped from above with a positive advantage: the bound's loss, no gradient
    o = O.policy_loss(z, a, lp - 1.0, np.abs(adv), None, w)
    assert np.allclose(o["row_loss"], -1.2 * w * np.abs(adv))
    assert not o["grad"].any() and np.isclose(o["totals"][4], w.sum())
    # uniform logits: entropy log n, over the legal ones only
    o = O.policy_loss(np.zeros((2, 9)), [0, 1], [0., 0.], [1., 1.], legal=[9, 4])
    assert np.allclose(o["entropy"], np.log([9, 4])) and not o["grad"][1, 4:].any()


def test_sequence_gradient_is_the_loss_difference():
    rng = np.random.default_rng(3)
    cu = O.cu_from_counts([9, 1, 6])
    s = rng.standard_normal(int(cu[-1])) * 2
    order = np.array([[3, 0, 7, 2], [-1] * 4, [4, 3, -1, -1]])
    k = [4, 0, 2]
    lp = [O.pl_logprob(s[cu[i] + 1:cu[i + 1]], order[i, :k[i]]) for i in range(3)]
    old, ref, adv = np.array(lp) - 0.1, np.array(lp) + 0.2, np.array([1.3, 1.0, -0.4])
    f = lambda x: O.pl_policy_loss(x, cu, k, order, old, adv, ref,  # noqa: E731
                                   kl_coef=0.3)["row_loss"].sum()
    grad = O.pl_policy_loss(s, cu, k, order, old, adv, ref, kl_coef=0.3)["grad"]
    for j in range(len(s)):
        e = np.zeros_like(s)
        e[j] = 1e-6
        assert abs((f(s + e) - f(s - e)) / 2e-6 - grad[j]) < 1e-7


def test_norm_and_adam_closed_forms():
    norm, f = O.grad_norm([np.full(9, 1e30, np.float32), np.zeros(0), np.full(16, 1e30)], 2.5e30)
    assert np.isclose(norm, 5e30, rtol=1e-7) and np.isclose(f, 0.5, rtol=1e-7)
    assert O.grad_norm([np.zeros(4)], 1.0) == (0.0, 1.0)
    # the first step from zero moments moves every weight by lr against the gradient's sign
    g = np.array([3.0, -0.2, 1e-3])
    p, m, v = O.adam_step(np.zeros(3), np.zeros(3), np.zeros(3), g, 1, 0.01, 0.9, 0.999, 0.0, 0.0)
    assert np.allclose(p, -0.01 * np.sign(g)) and np.allclose(m, 0.1 * g)
    # no gradient and no moments: only the decay is left
    p, _, _ = O.adam_step(np.ones(2), np.zeros(2), np.zeros(2), np.zeros(2), 5, 0.1, 0.9, 0.999,
                          1e-8, 0.5)
    assert np.allclose(p, 0.95)


@pytest.fixture(scope="module")
def lib():
    G.build()
    return P.load_library()


def test_policy_loss_host_checks(lib):
    f = ctypes.c_float
    good = [16, 2, 4, 8, 8, None, 16, 16, None, 16, None, f(.2), f(.2), f(0), f(0), 16, None, None,
            None, None, None, 0, None, None]
    for at, v in ((0, None), (0, 18), (1, 3), (1, -1), (2, -1), (3, 0), (4, 7), (6, None),
                  (7, None), (9, None), (11, f(-.1)), (11, f(1.5)), (12, f(-1)),
                  (12, f(float("inf"))), (13, f(float("nan"))), (13, f(.1)), (15, None),
                  (18, 17), (19, 16)):
        bad = list(good)
        bad[at] = v
        assert lib.dora_policy_loss(*bad) == 1, (at, v)
    good[19:22] = [16, 256, lib.dora_policy_workspace_size() - 1]     # workspace too small
    assert lib.dora_policy_loss(*good) == 1
    good[20:22] = [264, 1 << 20]                                      # and not aligned
    assert lib.dora_policy_loss(*good) == 1


def test_policy_loss_refuses_rows_that_32_bit_indexes_do_not_hold(lib):
    f = ctypes.c_float
    args = [16, 0, 1, (1 << 30) + 1, 1 << 40, None, 16, 16, None, 16, None, f(.2), f(.2), f(0),
            f(0), 16, None, None, None, None, None, 0, None, None]
    for classes in ((1 << 30) + 1, (1 << 31) - 1):
        args[3] = classes
        assert lib.dora_policy_loss(*args) == 1


def test_pl_policy_loss_host_checks(lib):
    f = ctypes.c_float
    good = [16, 16, 4, 100, 16, 16, 8, 16, None, 16, None, f(.2), f(.2), f(0), 16, None, None,
            None, None, 0, None, None]
    for at, v in ((0, None), (1, None), (2, -1), (3, -1), (4, None), (5, None), (6, 0), (6, 4096),
                  (7, None), (9, None), (11, f(2)), (13, f(.1)), (14, None), (17, 16)):
        bad = list(good)
        bad[at] = v
        assert lib.dora_pl_policy_loss(*bad) == 1, (at, v)


def test_param_list_host_checks(lib):
    def size(**kw):
        d = dict(grad=16, clipped=None, param=None, exp_avg=None, exp_avg_sq=None, copy=None,
                 n=10, grad_dtype=2, param_dtype=2)
        d.update(kw)
        return lib.dora_param_list_size(ctypes.byref(P._ParamC(**d)), 1)

    assert size() > 0 and size(n=0, grad=None) > 0
    assert size(param=16, exp_avg=16, exp_avg_sq=16, copy=16) > 0
    for bad in (dict(grad=None), dict(grad=18), dict(grad=17, grad_dtype=0), dict(clipped=18),
                dict(n=-1), dict(grad_dtype=3), dict(param=16), dict(param=16, exp_avg=16),
                dict(param=16, exp_avg=16, exp_avg_sq=16, param_dtype=7),
                dict(param=18, exp_avg=16, exp_avg_sq=16),
                dict(param=16, exp_avg=16, exp_avg_sq=16, copy=17)):
        assert size(**bad) == 0, bad
    c = P._ParamC(grad=16, n=10, grad_dtype=2, param_dtype=2)
    out = P._ParamListC()
    ok = lib.dora_param_list_size(ctypes.byref(c), 1)
    assert lib.dora_param_list_size(None, 1) == 0
    assert lib.dora_param_list_size(ctypes.byref(c), 0) == 0
    for args in ((None, 1, 256, ok), (ctypes.byref(c), 0, 256, ok), (ctypes.byref(c), 1, None, ok),
                 (ctypes.byref(c), 1, 264, ok), (ctypes.byref(c), 1, 256, ok - 1)):
        assert lib.dora_param_list_prepare(*args, ctypes.byref(out), None) == 1


def test_update_host_checks(lib):
    d = ctypes.c_double
    l = P._ParamListC(data=256, elements=10, count=1, spans=1, has_params=1)
    assert lib.dora_grad_norm(None, 1.0, 16, None) == 1
    assert lib.dora_grad_norm(ctypes.byref(l), -1.0, 16, None) == 1
    assert lib.dora_grad_norm(ctypes.byref(l), float("nan"), 16, None) == 1
    assert lib.dora_grad_norm(ctypes.byref(l), 1.0, None, None) == 1
    assert lib.dora_clip_grads(ctypes.byref(l), 1.0, None, None) == 1
    good = [ctypes.byref(l), 256, d(1e-3), d(.9), d(.999), d(1e-8), d(0), None, None]
    for at, v in ((0, None), (1, None), (1, 264), (2, d(float("nan"))), (3, d(1.0)), (3, d(-.1)),
                  (4, d(1.0)), (5, d(-1)), (6, d(-1)), (6, d(float("inf")))):
        bad = list(good)
        bad[at] = v
        assert lib.dora_adam_step(*bad) == 1, (at, v)
    without = P._ParamListC(data=256, elements=10, count=1, spans=1, has_params=0)
    assert lib.dora_adam_step(ctypes.byref(without), *good[1:]) == 1
    assert lib.dora_adam_init(None, 0, d(.9), d(.999), None) == 1
    assert lib.dora_adam_init(256, -1, d(.9), d(.999), None) == 1
    assert lib.dora_adam_init(256, 0, d(1.), d(.999), None) == 1
    assert lib.dora_adam_state_size() == 64


def test_binding_rejects_wrong_arguments(lib):
    import torch
    z, a, f = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    with pytest.raises(TypeError):
        P.dora_policy_loss(z, a, f, f, f)
    with pytest.raises(TypeError):
        P.dora_pl_policy_loss(f, a, a, a, f, f, f)
    with pytest.raises(TypeError):
        P.ParamList([f])
    with pytest.raises(ValueError):
        P.ParamList([])
    with pytest.raises(ValueError):
        P.ParamList([f], params=[f])
    with pytest.raises(ValueError):
        P.ParamList([f], copies=[f])
    with pytest.raises(ValueError):
        P.ParamList([f], clipped=[f, f])
