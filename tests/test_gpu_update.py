"""The policy update end to end: the weights' gradients of one epoch against
the oracle's losses in 64 bits, the step that follows, and a task that has to be
learned."""
import numpy as np
import pytest
import torch

import __graft_entry__ as G
import oracle as O
import paper_2609_34325_gb300 as P
from helpers import dev
from paper_2609_34325_gb300 import update as U

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    G.build()
    P.load_library()
    torch.cuda.set_device(0)


def _np(t):
    return t.detach().double().cpu().numpy()


def test_one_epoch_matches_the_oracle():
    heads = U.HeadUpdate(64, 20, dev(), seed=3, epochs=1, max_norm=1e-3)
    task = U.RemovalTask(24, 44, 64, dev(), seed=4)
    r = heads.act(*task.batch())
    reward, lost = task.rewards(r)
    adv, oadv = U.normalised(reward), U.normalised(-lost)
    # the log-probabilities taken down are those of the policy that acted: ratio 1
    logits, scores = heads.forward(r.z_cls, r.z_tok)
    before = [_np(w) for w in heads.weights]
    heads.losses(r, adv, oadv)
    b = r.budgets.shape[0]
    share = np.full(b, 1.0 / b)
    one = O.policy_loss(_np(logits), r.budgets.cpu().numpy(), _np(r.budget_logp), _np(adv),
                        weights=share, legal=r.legal.cpu().numpy(), entropy_coef=0.01)
    cu = r.cu.cpu().numpy()
    two = O.pl_policy_loss(_np(scores)[:cu[-1]], cu, r.k.cpu().numpy(), r.order.cpu().numpy(),
                           _np(r.order_logp), _np(oadv), weights=share)
    assert int(heads.status.item()) == 0 and np.all(_np(r.k) == 2 * (_np(r.budgets) + 1))
    z, t = _np(r.z_cls), _np(r.z_tok)[:cu[-1]]
    # d logits are rounded to bf16 (2^-9 each) and their product with the features once
    # more; the selector's gradient is fp32
    dw = one["grad"].T @ z
    tol = 2.0 ** -7 * (np.abs(one["grad"]).T @ np.abs(z)) + 1e-7
    assert np.all(np.abs(_np(heads.grads[0]) - dw) <= tol)
    assert np.all(np.abs(_np(heads.grads[1]) - one["grad"].sum(0)) <=
                  2.0 ** -8 * np.abs(one["grad"]).sum(0) + 1e-7)
    ds = two["grad"] @ t
    assert np.all(np.abs(_np(heads.grads[2]) - ds) <= 1e-4 * (np.abs(two["grad"]) @ np.abs(t)))
    assert np.allclose(_np(heads.totals)[0], one["totals"], rtol=1e-4, atol=1e-5)
    # and the step on the clipped gradients
    heads.update(r, adv, oadv)
    norm, f = O.grad_norm([_np(g) for g in heads.grads], 1e-3)
    assert f < 1 and abs(float(heads.norm[0]) - norm) <= 1e-6 * norm
    for w, p, g, c in zip(heads.weights, before, heads.grads, heads.copies):
        want, _, _ = O.adam_step(p, 0 * p, 0 * p, _np(g), 1, heads.lr, 0.9, 0.999, 1e-8, 0.0, f)
        assert np.all(np.abs(_np(w) - want) <= 1e-6 * heads.lr * 10 + 2.0 ** -22 * np.abs(want))
        assert torch.equal(c, w.to(torch.bfloat16))


def test_images_too_small_for_any_budget_take_no_part():
    heads = U.HeadUpdate(64, 20, dev(), seed=5)
    cu = torch.tensor([0, 3, 6, 30], dtype=torch.int32, device=dev())
    z = torch.randn(30, 64, device=dev()).to(torch.bfloat16)
    r = heads.act(z[cu[:-1].long()], z, cu)
    assert r.budgets[:2].tolist() == [-1, -1] and r.k[:2].tolist() == [0, 0]
    assert r.budget_logp[:2].tolist() == [0.0, 0.0] and r.order_logp[:2].tolist() == [0.0, 0.0]
    heads.update(r, torch.ones(3, device=dev()), torch.ones(3, device=dev()))
    assert int(heads.status.item()) == 0
    assert all(bool(torch.isfinite(w).all()) for w in heads.weights)


def test_the_task_is_learned():
    h = U.main(["--updates", "40", "--images", "128", "--tokens", "64", "--features", "64"])
    first, last = h[:3].mean(0).tolist(), h[-3:].mean(0).tolist()
    # importance is symmetric around 0.5 at random; a selector that has found the direction
    # removes the unimportant, and with them more of the tokens is worth its price
    assert abs(first[1] - 0.5) < 0.08
    assert last[1] < 0.35 and last[0] > first[0] + 0.1
