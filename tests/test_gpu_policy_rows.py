"""The categorical policy loss where every warp, CTA or cluster has several rows,
at each way that a row can be held, against the formulas in 64 bits.

Rows start at any alignment (an odd pitch), the legal logits end anywhere in them
(NaN past them and between rows), some rows take no part.  The bounds are those of
test_gpu_policy.py: log-probabilities to LOGP times (2 + their size + the logarithm
of the sum), every other value to as much of the terms that it sums, and a result in
16 bits to one rounding more."""
import math

import numpy as np
import pytest
import torch

import __graft_entry__ as G
import oracle as O
import paper_2609_34325_gb300 as P
from helpers import dev

LOGP = 2e-6
KL, ENT, LOW, HIGH = 0.05, 0.01, 0.2, 0.2
BF16, F16, F32, F64 = torch.bfloat16, torch.float16, torch.float32, torch.float64
ELEMS = {BF16: 8, F16: 8, F32: 4}                          # of 16 bytes
ROUND = {BF16: (2.0 ** -8, 0.0), F16: (2.0 ** -11, 2.0 ** -24), F32: (0.0, 0.0)}


def _reference(z, legal, actions, old, ref, adv, w):
    """logp, entropy, row_loss, grad and totals in 64 bits; rows without an action or
    of weight 0 are 0."""
    classes = z.shape[1]
    past = torch.arange(classes, device=z.device)[None] >= legal[:, None]
    live = (actions >= 0) & (w != 0)
    z = z.to(F64).masked_fill(past, -math.inf)
    lq = torch.where(past, 0.0, z - z.logsumexp(1, keepdim=True))
    p = torch.where(past, 0.0, lq.exp())
    del z
    at = actions.clamp(min=0).long()[:, None]
    logp = lq.gather(1, at)[:, 0]
    h = -(p * lq).sum(1)
    rho = (logp - old).exp()
    plain, cut = rho * adv, rho.clamp(1 - LOW, 1 + HIGH) * adv
    clipped = plain > cut
    x = ref - logp
    pol, kl = -torch.where(clipped, cut, plain), x.expm1() - x
    g = w * (torch.where(clipped, 0.0, -plain) - KL * x.expm1())
    loss = w * (pol + KL * kl - ENT * h)
    grad = p * (w * ENT)[:, None] * (lq + h[:, None]) - g[:, None] * p
    grad.scatter_add_(1, at, g[:, None])
    terms = torch.stack([loss, w * pol, w * kl, w * h, w * clipped, w])
    return {"logp": torch.where(live, logp, 0.0), "entropy": torch.where(live, h, 0.0),
            "row_loss": torch.where(live, loss, 0.0),
            "grad": torch.where(live[:, None] & ~past, grad, 0.0),
            "totals": torch.where(live, terms, 0.0).sum(1)}, live


def _inputs(rows, classes, dtype, seed, device):
    """Logits and the rows' scalars: ratios on both sides of each clipping bound, none
    within 1e-3 of it."""
    g = torch.Generator().manual_seed(seed)
    z = torch.empty(rows, classes, device=device)
    z.normal_(0.0, 2.5, generator=torch.Generator(device=device).manual_seed(seed))
    z = z.to(dtype)
    legal = torch.randint(1, classes + 1, (rows,), generator=g)
    legal[::5] = classes
    legal[1::11] = torch.randint(1, min(classes, 20) + 1, legal[1::11].shape, generator=g)
    actions = (torch.rand(rows, generator=g) * legal).long().clamp(max=classes - 1)
    w = torch.rand(rows, generator=g) + 0.1
    out = torch.rand(rows, generator=g) < 0.15
    actions[out & (torch.arange(rows) % 2 == 0)] = -1
    w[out & (torch.arange(rows) % 2 == 1)] = 0.0
    legal, actions, w = (t.to(device) for t in (legal, actions, w))
    none = torch.zeros(rows, dtype=F64, device=device)
    lp = _reference(z, legal, actions.clamp(min=0), none, none, none, none + 1)[0]["logp"]
    delta = torch.tensor([0.01, 0.1, -0.1, 0.3, -0.4, -0.02, 0.5], device=device)
    old = (lp - delta.repeat(rows // 7 + 1)[:rows]).float()
    ref = (lp + 0.2 * torch.randn(rows, generator=g).to(device)).float()
    adv = torch.randn(rows, generator=g).to(device)
    return z, legal, actions, old, ref, adv, w


def test_the_64_bit_form_is_the_oracles():
    z, legal, actions, old, ref, adv, w = _inputs(40, 23, F32, 1, "cpu")
    got, _ = _reference(z, legal, actions, old.to(F64), ref.to(F64), adv.to(F64), w.to(F64))
    want = O.policy_loss(z.double().numpy(), actions.numpy(), old.numpy(), adv.numpy(),
                         ref.numpy(), w.numpy(), legal.numpy(), LOW, HIGH, KL, ENT)
    for n in want:
        assert np.allclose(got[n].numpy(), want[n], rtol=1e-11, atol=1e-12), n


@pytest.fixture(scope="module")
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    G.build()
    P.load_library()
    torch.cuda.set_device(0)


def _near(got, want, tol, what):
    got = got.to(F64)
    assert bool(torch.isfinite(got).all()), what
    over = (got - want).abs() - tol
    assert float(over.max()) <= 0, (what, float(over.max()))


def _run(z, classes, q, grad):
    rows = z.shape[0]
    out = {n: torch.full((rows,), 7.0, device=dev()) for n in ("logp", "entropy", "row_loss")}
    out["totals"] = torch.full((6,), 7.0, device=dev())
    st = torch.zeros(1, dtype=torch.int32, device=dev())
    P.dora_policy_loss(z, q["actions"], q["old"], q["adv"], out["logp"],
                       P.alloc_policy_workspace(dev()), grad=grad, classes=classes,
                       legal=q["legal"], ref_logp=q["ref"], weights=q["w"], clip_low=LOW,
                       clip_high=HIGH, kl_coef=KL, entropy_coef=ENT, entropy=out["entropy"],
                       row_loss=out["row_loss"], totals=out["totals"], status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    return out


# 16-byte granules a row and rows: 8 and 32 lanes a row (to 32 and 512 granules), a CTA a
# row (to 2048, and up to 512 where rows are few), one CTA, and clusters of 2, 4 and 8,
# with a ring (to 4096 a CTA), and rows longer than eight CTAs' rings
ROWS = [(5, 39500), (24, 39500), (100, 9900), (200, 9900), (400, 9900), (400, 700), (800, 2500),
        (1500, 1300), (3000, 700), (6000, 400), (12000, 200), (20000, 100), (34000, 80)]


@pytest.mark.gpu
@pytest.mark.parametrize("odd", [0, 1])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("granules,rows", ROWS)
def test_several_rows_a_team(granules, rows, dtype, odd, _built):
    # aligned rows that are used whole, and rows that start and end inside a granule
    classes = granules * ELEMS[dtype] - 3 * odd
    pitch = classes + 2 * odd
    z0, legal, actions, old, ref, adv, w = _inputs(rows, classes, dtype, granules + odd, dev())
    want, live = _reference(z0, legal, actions, old.to(F64), ref.to(F64), adv.to(F64), w.to(F64))
    z = torch.full((rows, pitch), math.nan, dtype=dtype, device=dev())
    z[:, :classes] = z0.masked_fill(
        torch.arange(classes, device=dev())[None] >= legal[:, None], math.nan)
    del z0
    q = dict(legal=legal.int(), actions=actions.int(), old=old, ref=ref, adv=adv, w=w)
    grad = torch.full_like(z, 7.0)
    out = _run(z, classes, q, grad)

    w = w.to(F64)
    rel = LOGP * (2 + want["logp"].abs() + math.log(classes))
    a = adv.to(F64).abs() * 2 + KL * 2 + ENT * math.log(classes) + 1e-3
    _near(out["logp"], want["logp"], rel, "logp")
    _near(out["entropy"], want["entropy"],
          torch.full_like(rel, LOGP * (4 + math.log(classes))), "entropy")
    _near(out["row_loss"], want["row_loss"], w * a * rel, "row_loss")
    tot = (w * a * rel).sum() + (w * (1 + math.log(classes)) * rel).sum()
    _near(out["totals"], want["totals"], tot + 1e-7, "totals")
    assert bool((grad[:, classes:] == 7.0).all())
    r, c = ROUND[dtype]
    term = (w * a * rel)[:, None]
    size = want["grad"].abs()
    _near(grad[:, :classes], want["grad"],
          torch.minimum(term, rel[:, None] * size + 0.02 * term) + r * size + c, "grad")
    assert not grad[:, :classes][~live].any()

    # without the gradient, and with the gradient over the logits: the same bits
    again = _run(z, classes, q, None)
    over = _run(z, classes, q, z)
    for n in out:
        assert torch.equal(out[n], again[n]) and torch.equal(out[n], over[n]), n
    assert torch.equal(z[:, :classes], grad[:, :classes])
