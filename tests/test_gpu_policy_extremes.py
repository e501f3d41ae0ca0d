"""Ratios and KL terms past fp32's range, in both policy losses.

Where a term is left out (its coefficient or the advantage is 0) the bound is that
of the same call without it: the same bits.  Infinite terms are compared as such."""
import math

import numpy as np
import pytest
import torch

import __graft_entry__ as G
import oracle as O
import paper_2609_34325_gb300 as P
from helpers import dev, f32, i32


@pytest.fixture(scope="module")
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    G.build()
    P.load_library()
    torch.cuda.set_device(0)


def _rows(classes, far):
    """Six rows; in row 2 and 4 the action's logit lies `far` below the others."""
    rng = np.random.default_rng(classes)
    z = rng.standard_normal((6, classes)).astype(np.float32)
    actions = rng.integers(0, classes, 6)
    z[2, actions[2]] = z[4, actions[4]] = far
    lp = np.array([O.log_softmax(z[r].astype(np.float64))[actions[r]] for r in range(6)])
    return z, actions, lp


def _policy(z, actions, old, adv, **kw):
    out = {n: torch.full((6,), 7.0, device=dev()) for n in ("logp", "row_loss", "totals")}
    out["grad"] = torch.full(z.shape, 7.0, device=dev())
    P.dora_policy_loss(f32(z), i32(actions), f32(old), f32(adv), out["logp"],
                       P.alloc_policy_workspace(dev()), grad=out["grad"],
                       row_loss=out["row_loss"], totals=out["totals"], **kw)
    return out


def _images(far):
    """Three images; in image 1 the second token to be removed lies `far` below."""
    cu, k, order = np.array([0, 6, 12, 18]), np.array([2, 3, 2]), np.array([[1, 0, -1], [2, 0, 3],
                                                                            [4, 1, -1]])
    s = np.random.default_rng(3).standard_normal(18).astype(np.float32)
    s[7] = far
    lp = np.array([O.pl_logprob(s[cu[i] + 1:cu[i + 1]].astype(np.float64), order[i, :k[i]])
                   for i in range(3)])
    return s, cu, k, order, lp


def _sequences(s, cu, k, order, old, adv, **kw):
    out = {"logp": torch.full((3,), 7.0, device=dev()),
           "row_loss": torch.full((3,), 7.0, device=dev()),
           "totals": torch.full((6,), 7.0, device=dev()),
           "grad": torch.full((len(s),), 7.0, device=dev())}
    P.dora_pl_policy_loss(f32(s), i32(cu), i32(k), i32(order), f32(old), f32(adv), out["logp"],
                          P.alloc_policy_workspace(dev()), grad=out["grad"],
                          row_loss=out["row_loss"], totals=out["totals"], **kw)
    return out


def test_oracle_leaves_out_a_kl_term_of_coefficient_zero():
    args = (np.array([[0., -800., 1.]]), [1], [-801.3], [2.0])
    a, b = O.policy_loss(*args, ref=[-0.5]), O.policy_loss(*args)
    assert a["totals"][2] == np.inf and b["totals"][2] == 0
    for n in ("logp", "row_loss", "grad"):
        assert np.isfinite(a[n]).all() and np.array_equal(a[n], b[n])


@pytest.mark.gpu
@pytest.mark.parametrize("classes", [50, 1500, 20000, 140000])
def test_a_kl_term_of_coefficient_zero_is_only_reported(classes, _built):
    z, actions, lp = _rows(classes, -200.0)                # exp(ref - logp) is past fp32
    old, adv, ref = lp - 0.1, np.linspace(-1, 1, 6), np.full(6, -0.5)
    a = _policy(z, actions, old, adv, ref_logp=f32(ref), kl_coef=0.0)
    b = _policy(z, actions, old, adv)
    for n in ("logp", "row_loss", "grad"):
        assert bool(torch.isfinite(a[n]).all()) and torch.equal(a[n], b[n]), n
    assert torch.equal(a["totals"][:2], b["totals"][:2]) and float(a["totals"][2]) == math.inf
    assert float(_policy(z, actions, old, adv, ref_logp=f32(ref), kl_coef=0.1)["row_loss"][2]) \
        == math.inf


@pytest.mark.gpu
def test_a_kl_term_of_coefficient_zero_is_only_reported_of_sequences(_built):
    s, cu, k, order, lp = _images(-150.0)
    old, adv, ref = lp - 0.1, np.array([1.0, -1.0, 0.5]), np.full(3, -0.5)
    a = _sequences(s, cu, k, order, old, adv, ref_logp=f32(ref), kl_coef=0.0)
    b = _sequences(s, cu, k, order, old, adv)
    for n in ("logp", "row_loss", "grad"):
        assert bool(torch.isfinite(a[n]).all()) and torch.equal(a[n], b[n]), n
    assert torch.equal(a["totals"][:2], b["totals"][:2]) and float(a["totals"][2]) == math.inf


def test_oracle_kl_of_an_action_of_probability_zero():
    o = O.policy_loss(np.array([[0., -np.inf, 1.]]), [1], [-1.0], [2.0], ref=[-0.5], kl_coef=0.1)
    assert o["logp"][0] == -np.inf and o["row_loss"][0] == np.inf and o["totals"][2] == np.inf


@pytest.mark.gpu
@pytest.mark.parametrize("classes", [50, 1500, 20000, 140000])
def test_kl_of_an_action_of_probability_zero(classes, _built):
    z, actions, lp = _rows(classes, -math.inf)
    old, adv, ref = np.where(np.isinf(lp), -1.0, lp), np.linspace(-1, 1, 6), np.full(6, -0.5)
    bad = np.isinf(lp)
    out = _policy(z, actions, old, adv, ref_logp=f32(ref), kl_coef=0.1)
    loss = out["row_loss"].cpu().numpy()
    assert np.all(out["logp"].cpu().numpy()[bad] == -np.inf)
    assert np.all(loss[bad] == np.inf) and np.isfinite(loss[~bad]).all()
    assert float(out["totals"][0]) == math.inf and float(out["totals"][2]) == math.inf
    assert not np.isfinite(out["grad"].cpu().numpy()[bad, actions[bad]]).any()
    assert bool(torch.isfinite(out["grad"].cpu()[torch.from_numpy(~bad)]).all())
    # where the term is only reported, the ratio 0 has its clipped loss and no gradient
    out = _policy(z, actions, old, adv, ref_logp=f32(ref), kl_coef=0.0)
    assert bool(torch.isfinite(out["grad"]).all()) and float(out["totals"][2]) == math.inf
    want = np.where(adv < 0, -0.8 * adv, 0.0)
    assert np.allclose(out["row_loss"].cpu().numpy()[bad], want[bad], rtol=1e-6, atol=0)
    assert not out["grad"].cpu().numpy()[bad].any()


@pytest.mark.gpu
def test_kl_of_a_sequence_of_probability_zero(_built):
    s, cu, k, order, lp = _images(-math.inf)
    assert lp[1] == -np.inf
    old, adv, ref = np.where(np.isinf(lp), -1.0, lp), np.ones(3), np.full(3, -0.5)
    out = _sequences(s, cu, k, order, old, adv, ref_logp=f32(ref), kl_coef=0.1)
    assert float(out["row_loss"][1]) == math.inf and bool(torch.isfinite(out["row_loss"][::2]).all())
    assert float(out["totals"][0]) == math.inf and float(out["totals"][2]) == math.inf


@pytest.mark.gpu
@pytest.mark.parametrize("classes", [50, 1500, 20000, 140000])
def test_an_advantage_of_zero_has_no_policy_term_at_any_ratio(classes, _built):
    z, actions, lp = _rows(classes, 3.0)
    old = lp - 0.1
    old[1:3] = -300.0                                      # the ratio is past fp32
    o = O.policy_loss(z, actions, old, np.zeros(6), entropy_coef=0.01)
    out = _policy(z, actions, old, np.zeros(6), entropy_coef=0.01)
    assert not o["totals"][1] and not out["totals"][1:2].any()
    assert np.allclose(out["row_loss"].cpu().numpy(), o["row_loss"], rtol=1e-5, atol=0)
    assert np.all(np.abs(out["grad"].cpu().numpy() - o["grad"]) <= 1e-6)
    # a ratio that is no number is not hidden
    assert math.isnan(float(_policy(z, actions, np.full(6, np.nan), np.zeros(6))["row_loss"][0]))


@pytest.mark.gpu
def test_an_advantage_of_zero_has_no_policy_term_of_sequences(_built):
    s, cu, k, order, lp = _images(1.0)
    out = _sequences(s, cu, k, order, np.full(3, -300.0), np.zeros(3))
    assert not out["row_loss"].any() and not out["grad"].any() and not out["totals"][:3].any()
