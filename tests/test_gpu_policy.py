"""GPU parity of the policy update through the C ABI, against the fp64 oracle.

Bounds.  The losses compute in fp32: a logit difference to the row's maximum
carries 2^-24 of its size, an exponential a few 2^-23 of its value, and a
logarithm of the sum 2^-23 of its own, so that log-probabilities are good to
LOGP times (2 + their size) and ratios, and with them losses and gradients, to
that much relatively, plus as much of every term they sum.  A result in 16 bits
is rounded once more: 2^-9 (bf16) or 2^-12 (fp16, and 2^-25 absolute) of it."""
import numpy as np
import pytest
import torch

import __graft_entry__ as G
import oracle as O
import paper_2609_34325_gb300 as P
from helpers import dev, f32, i32

pytestmark = pytest.mark.gpu

LOGP = 2e-6
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
HALF_ULP = {BF16: (2.0 ** -8, 0.0), F16: (2.0 ** -11, 2.0 ** -24), F32: (0.0, 0.0)}


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    G.build()
    P.load_library()
    torch.cuda.set_device(0)


def _status():
    return torch.zeros(1, dtype=torch.int32, device=dev())


def _near(got, ref, tol, what):
    got, ref = np.asarray(got, dtype=np.float64), np.asarray(ref, dtype=np.float64)
    err = np.abs(got - ref)
    assert np.isfinite(got).all(), what
    assert np.all(err <= tol), (what, float(np.max(err - tol)), float(err.max()))


class _Case:
    """One call's inputs on the host (fp32 arrays; logits already rounded)."""

    def __init__(self, rows, classes, dtype, seed, legal=False, idle=0.0, ref=True, weights=True,
                 pitch=0, std=2.5, kl=0.05, ent=0.01):
        rng = np.random.default_rng(seed)
        self.dtype, self.kl, self.ent = dtype, kl if ref else 0.0, ent
        self.pitch = pitch or classes
        t = torch.from_numpy((rng.standard_normal((rows, classes)) * std).astype(np.float32))
        self.z = t.to(dtype).double().numpy()
        self.legal = rng.integers(1, classes + 1, rows) if legal else None
        n = self.legal if legal else np.full(rows, classes)
        self.actions = (rng.random(rows) * n).astype(np.int64)
        lp = np.array([O.log_softmax(self.z[r, :n[r]])[self.actions[r]] for r in range(rows)])
        # ratios on both sides of each clipping bound, none within 1e-3 of it
        delta = np.tile([0.01, 0.1, -0.1, 0.3, -0.4, -0.02, 0.5], rows)[:rows]
        self.old = (lp - delta).astype(np.float32)
        self.ref = (lp + 0.2 * rng.standard_normal(rows)).astype(np.float32) if ref else None
        self.adv = rng.standard_normal(rows).astype(np.float32)
        self.w = (rng.random(rows) + 0.1).astype(np.float32) if weights else None
        out = rng.random(rows) < idle
        if idle:
            self.actions[out & (np.arange(rows) % 2 == 0)] = -1
            if weights:
                self.w[out & (np.arange(rows) % 2 == 1)] = 0.0

    def device(self, fill=np.nan):
        rows, classes = self.z.shape
        full = torch.full((rows, self.pitch), fill, dtype=torch.float64)
        full[:, :classes] = torch.from_numpy(self.z)
        if self.legal is not None:
            full[:, :classes][torch.arange(classes)[None] >=
                              torch.from_numpy(self.legal)[:, None]] = fill
        return full.to(self.dtype).to(dev())

    def run(self, logits=None, grad=None, stream=None, want_grad=True):
        rows, classes = self.z.shape
        z = self.device() if logits is None else logits
        out = {n: torch.full((rows,), 7.0, device=dev()) for n in ("logp", "entropy", "row_loss")}
        out["totals"] = torch.full((6,), 7.0, device=dev())
        out["grad"] = (torch.full_like(z, 7.0) if grad is None else grad) if want_grad else None
        st = _status()
        opt = lambda a, f: None if a is None else f(a)  # noqa: E731
        args = (i32(self.actions), f32(self.old), f32(self.adv))
        kw = dict(legal=opt(self.legal, i32), ref_logp=opt(self.ref, f32),
                  weights=opt(self.w, f32))
        ws = P.alloc_policy_workspace(dev())
        torch.cuda.synchronize()
        P.dora_policy_loss(z, *args, out["logp"], ws, grad=out["grad"], classes=classes,
                           kl_coef=self.kl, entropy_coef=self.ent, entropy=out["entropy"],
                           row_loss=out["row_loss"], totals=out["totals"], status=st,
                           stream=stream, **kw)
        torch.cuda.synchronize()
        assert int(st.item()) == 0
        return out

    def check(self, out, rows=None):
        o = O.policy_loss(self.z, self.actions, self.old, self.adv, self.ref, self.w, self.legal,
                          kl_coef=self.kl, entropy_coef=self.ent)
        classes = self.z.shape[1]
        w = np.ones(len(self.old)) if self.w is None else self.w
        rel = LOGP * (2 + np.abs(o["logp"]) + np.log(classes))
        a = np.abs(self.adv) * 2 + self.kl * 2 + self.ent * np.log(classes) + 1e-3
        _near(out["logp"].cpu(), o["logp"], rel, "logp")
        _near(out["entropy"].cpu(), o["entropy"], LOGP * (4 + np.log(classes)), "entropy")
        _near(out["row_loss"].cpu(), o["row_loss"], w * a * rel, "row_loss")
        tot = (w * a * rel).sum() + (w * (1 + np.log(classes)) * rel).sum()
        _near(out["totals"].cpu(), o["totals"], tot + 1e-7, "totals")
        if out["grad"] is not None:
            r, c = HALF_ULP[self.dtype]
            got = out["grad"][:, :classes].double().cpu().numpy()
            # g (1 - p) near p = 1 and p (log p + H) cancel: the bound is of their terms
            term = (w * a * rel)[:, None]
            p = np.abs(o["grad"])
            _near(got, o["grad"], np.minimum(term, rel[:, None] * p + 0.02 * term) + r * p + c, "grad")


SHAPES = [(1, 1), (1, 2), (3, 1), (5, 7), (64, 96), (9, 64), (33, 65), (4, 255), (7, 1000),
          (2, 1025), (3, 4097), (3, 9001), (2, 16390), (1, 33333), (2, 70001)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,classes", SHAPES)
def test_policy_loss_shapes(rows, classes, dtype):
    c = _Case(rows, classes, dtype, rows * 100003 + classes)
    c.check(c.run())


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("classes,pitch", [(96, 97), (1000, 1024), (333, 337), (5003, 5005),
                                           (17000, 17001)])
def test_policy_loss_masks_pitches_and_idle_rows(classes, pitch, dtype):
    # legal prefixes with NaN past them and between rows, a third of the rows idle
    c = _Case(41, classes, dtype, classes, legal=True, idle=0.35, pitch=pitch)
    z = c.device()
    grad = torch.full_like(z, 7.0)
    out = c.run(z, grad)
    c.check(out)
    assert bool((grad[:, classes:] == 7.0).all())          # past the classes: not written
    past = torch.arange(classes, device=dev())[None] >= i32(c.legal)[:, None]
    assert bool((grad[:, :classes][past] == 0).all())
    idle = c.actions < 0
    if c.w is not None:
        idle = idle | (c.w == 0)
    assert idle.any() and not out["logp"].cpu().numpy()[idle].any()
    assert not out["grad"][:, :classes].cpu()[torch.from_numpy(idle)].any()


@pytest.mark.parametrize("classes", [100, 3001, 40001])
def test_policy_loss_options(classes):
    c = _Case(6, classes, BF16, 5, ref=False, weights=False, ent=0.0)
    c.check(c.run())
    c = _Case(6, classes, F32, 6)
    out = c.run(want_grad=False)                           # forward only
    c.check(out)
    assert out["grad"] is None
    z = c.device()
    inplace = c.run(z, z)                                  # the gradient over the logits
    c.check(inplace)
    for n in ("logp", "entropy", "row_loss", "totals"):
        assert torch.equal(inplace[n], out[n])
    z = c.device()
    logp = torch.zeros(6, device=dev())
    P.dora_policy_loss(z, i32(c.actions), f32(c.old), f32(c.adv), logp)   # logp alone
    assert torch.equal(logp, out["logp"])


@pytest.mark.parametrize("classes", [96, 2050, 50001])
def test_policy_loss_same_bits_and_other_streams(classes):
    c = _Case(300 if classes < 50000 else 20, classes, F32, 9, idle=0.2)
    a, b = c.run(), c.run()
    side = torch.cuda.Stream()
    d = c.run(stream=side)
    for n in a:
        assert torch.equal(a[n], b[n]) and torch.equal(a[n], d[n]), n


@pytest.mark.parametrize("classes", [50, 1500, 20000])
def test_policy_loss_lowest_values_and_infinities(classes):
    c = _Case(5, classes, F32, 11, std=1.0)
    z = c.device()
    lowest = torch.finfo(torch.float32).min
    keep = torch.zeros(5, classes, dtype=torch.bool)
    keep[:, ::3] = True
    keep[torch.arange(5), torch.from_numpy(c.actions)] = True
    for value in (lowest, -np.inf):                        # actions of probability 0
        zz = torch.where(keep.to(dev()), z, value)
        c.z = zz.double().cpu().numpy()
        ref = np.where(keep.numpy(), c.z, -np.inf)
        out = c.run(zz)
        o = O.policy_loss(ref, c.actions, c.old, c.adv, c.ref, c.w, kl_coef=c.kl,
                          entropy_coef=c.ent)
        # old log-probabilities are those of the unmasked rows: ratios of some size
        scale = np.exp(np.abs(o["logp"] - c.old)) * 10
        _near(out["logp"].cpu(), o["logp"], 1e-5 * (1 + np.abs(o["logp"])), "logp")
        got = out["grad"].double().cpu().numpy()
        assert np.all(got[~keep.numpy()] == 0)
        _near(got, o["grad"], 1e-5 * scale[:, None], "grad")
    # one certain action: probability 1, no entropy, no gradient left
    zz = torch.full_like(z, lowest)
    zz[torch.arange(5), torch.from_numpy(c.actions).to(dev())] = 3.0
    out = c.run(zz)
    assert torch.equal(out["logp"], torch.zeros_like(out["logp"]))
    assert torch.equal(out["entropy"], torch.zeros_like(out["entropy"]))
    assert not out["grad"].any()


@pytest.mark.parametrize("classes", [50, 1500, 20000, 70000])
def test_policy_loss_nan_rows_stay_in_their_rows(classes):
    c = _Case(6, classes, F32, 12)
    z = c.device()
    clean = c.run(z.clone())
    z[1, classes // 2] = np.nan
    z[3, classes - 1] = np.inf
    z[4] = -np.inf
    st = _status()
    logp = torch.zeros(6, device=dev())
    grad = torch.zeros_like(z)
    tot, ws = torch.zeros(6, device=dev()), P.alloc_policy_workspace(dev())
    P.dora_policy_loss(z, i32(c.actions), f32(c.old), f32(c.adv), logp, ws, grad=grad,
                       ref_logp=f32(c.ref), weights=f32(c.w), kl_coef=c.kl, entropy_coef=c.ent,
                       totals=tot, status=st)
    torch.cuda.synchronize()
    bad = torch.tensor([False, True, False, True, True, False], device=dev())
    assert bool(torch.isnan(logp[bad]).all()) and bool(torch.isnan(grad[bad]).any(1).all())
    assert torch.equal(logp[~bad], clean["logp"][~bad])
    assert torch.equal(grad[~bad], clean["grad"][~bad])
    assert bool(torch.isnan(tot[0]))


@pytest.mark.parametrize("classes", [12, 700, 9000, 70000])
def test_policy_loss_bad_actions(classes):
    c = _Case(5, classes, BF16, 13, legal=True)
    z = c.device(fill=0.0)
    c.actions[1] = c.legal[1]                              # past the legal ones
    c.legal[2] = classes + 1
    c.legal[3], c.actions[3] = 0, 0                        # nothing is legal
    c.legal[4], c.actions[4] = 0, -1                       # and no action taken: no part
    logp, ent = torch.zeros(5, device=dev()), torch.zeros(5, device=dev())
    grad, st = torch.zeros_like(z), _status()
    P.dora_policy_loss(z, i32(c.actions), f32(c.old), f32(c.adv), logp, grad=grad,
                       legal=i32(c.legal), entropy=ent, status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == O.DORA_ERR_DEVICE_BAD_COUNT
    assert torch.isnan(logp).tolist() == [False, True, True, True, False]
    assert torch.isnan(ent).tolist() == [False, True, True, True, False]
    assert bool(torch.isnan(grad[1:4]).all()) and not bool(torch.isnan(grad[0]).any())
    assert float(logp[4]) == 0 and not grad[4].any()


def test_policy_loss_empty_and_idle_batches():
    ws = P.alloc_policy_workspace(dev())
    tot = torch.full((6,), 3.0, device=dev())
    e, ei = torch.zeros(0, device=dev()), torch.zeros(0, dtype=torch.int32, device=dev())
    P.dora_policy_loss(torch.zeros(0, 40, device=dev()), ei, e, e, e, ws, totals=tot)
    assert not tot.any()
    for classes in (40, 4000):
        z = torch.full((9, classes), np.nan, device=dev())
        logp, grad = torch.ones(9, device=dev()), torch.ones_like(z)
        tot = torch.full((6,), 3.0, device=dev())
        P.dora_policy_loss(z, i32(np.full(9, -1)), f32(np.zeros(9)), f32(np.zeros(9)), logp, ws,
                           grad=grad, totals=tot, entropy_coef=0.1)
        assert not tot.any() and not logp.any() and not grad.any()


def test_policy_loss_offsets_past_32_bits():
    # 2.4e9 logits: the last rows lie past 2^31 elements
    rows, classes = 40000, 60000
    z = torch.zeros(rows, classes, dtype=BF16, device=dev())
    z[-3:] = torch.randn(3, classes, device=dev()).to(BF16)
    act = torch.full((rows,), -1, dtype=torch.int32, device=dev())
    act[-3:] = torch.tensor([0, 12345, classes - 1], dtype=torch.int32, device=dev())
    ref = z[-3:].double().cpu().numpy()
    lp = np.array([O.log_softmax(ref[i])[a] for i, a in enumerate((0, 12345, classes - 1))])
    old, adv = torch.zeros(rows, device=dev()), torch.ones(rows, device=dev())
    old[-3:] = f32(lp - 0.1)
    logp = torch.zeros(rows, device=dev())
    P.dora_policy_loss(z, act, old, adv, logp, grad=z)     # in place
    torch.cuda.synchronize()
    o = O.policy_loss(ref, [0, 12345, classes - 1], lp - 0.1, np.ones(3))
    _near(logp[-3:].cpu(), lp, 1e-4, "logp")
    _near(z[-3:].double().cpu(), o["grad"], 2.0 ** -8 * np.abs(o["grad"]) + 1e-4 * np.abs(o["grad"]),
          "grad")
    assert not logp[:-3].any() and not z[:-3].any()


def test_policy_loss_in_a_graph():
    c = _Case(64, 96, F32, 21, legal=True)
    want = c.run()
    z, ws = c.device(), P.alloc_policy_workspace(dev())
    out = {n: torch.zeros(64, device=dev()) for n in ("logp", "entropy", "row_loss")}
    grad, tot = torch.zeros_like(z), torch.zeros(6, device=dev())
    args = (i32(c.actions), f32(c.old), f32(c.adv))
    kw = dict(legal=i32(c.legal), ref_logp=f32(c.ref), weights=f32(c.w))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            P.dora_policy_loss(z, *args, out["logp"], ws, grad=grad, kl_coef=c.kl,
                               entropy_coef=c.ent, entropy=out["entropy"],
                               row_loss=out["row_loss"], totals=tot, **kw)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(tot, want["totals"]) and torch.equal(grad[:, :96], want["grad"][:, :96])


# ---------------------------------------------------------------------------
# ordered removals
# ---------------------------------------------------------------------------

def _orders(rng, scores, cu, k, k_cap):
    out = np.full((len(k), k_cap), -1, dtype=np.int64)
    for i in range(len(k)):
        n = int(cu[i + 1] - cu[i]) - 1
        if k[i]:
            s = scores[cu[i] + 1:cu[i + 1]]
            out[i, :k[i]] = np.argsort(-(s + rng.gumbel(size=n)), kind="stable")[:k[i]]
    return out


def _sequences(lens, k, std, seed, k_cap=None):
    rng = np.random.default_rng(seed)
    cu = O.cu_from_counts(lens)
    s = (rng.standard_normal(int(cu[-1])) * std).astype(np.float32)
    order = _orders(rng, s, cu, k, k_cap or max(1, max(k)))
    lp = np.array([O.pl_logprob(s[cu[i] + 1:cu[i + 1]], order[i, :k[i]]) if k[i] else 0.0
                   for i in range(len(k))])
    delta = np.tile([0.01, 0.1, -0.1, 0.3, -0.4, -0.02], len(k))[:len(k)]
    return (s, cu, np.asarray(k), order, (lp - delta).astype(np.float32),
            rng.standard_normal(len(k)).astype(np.float32),
            (lp + 0.2 * rng.standard_normal(len(k))).astype(np.float32),
            (rng.random(len(k)) + 0.1).astype(np.float32))


def _run_sequences(q, kl=0.05, weights=True, ref=True, grad=True, stream=None):
    s, cu, k, order, old, adv, rf, w = q
    b = len(k)
    out = {n: torch.full((b,), 7.0, device=dev()) for n in ("logp", "row_loss")}
    out["totals"] = torch.full((6,), 7.0, device=dev())
    out["grad"] = torch.full((len(s) + 5,), 7.0, device=dev()) if grad else None
    sc = torch.full((len(s) + 5,), np.nan, device=dev())
    sc[:len(s)] = f32(s)
    st, ws = _status(), P.alloc_policy_workspace(dev())
    args = (i32(cu), i32(k), i32(order), f32(old), f32(adv))
    rf, w = f32(rf) if ref else None, f32(w) if weights else None
    torch.cuda.synchronize()
    P.dora_pl_policy_loss(sc, *args, out["logp"], ws, grad=out["grad"], ref_logp=rf, weights=w,
                          kl_coef=kl if ref else 0.0, row_loss=out["row_loss"],
                          totals=out["totals"], status=st, stream=stream)
    torch.cuda.synchronize()
    return out, int(st.item())


def _check_sequences(q, out, kl=0.05, weights=True, ref=True):
    s, cu, k, order, old, adv, rf, w = q
    o = O.pl_policy_loss(s, cu, k, order, old, adv, rf if ref else None, w if weights else None,
                         kl_coef=kl if ref else 0.0)
    w = w if weights else np.ones(len(k))
    # a step's term carries LOGP of its size; k of them are summed
    size = 2 + np.abs(s).max() + np.log(np.diff(cu).max() + 1)
    rel = 1e-6 + LOGP * k * size / np.maximum(1, np.sqrt(k)) + 2.0 ** -22
    a = np.abs(adv) * 2 + kl * 2
    _near(out["logp"].cpu(), o["logp"], rel + 2.0 ** -23 * np.abs(o["logp"]), "logp")
    _near(out["row_loss"].cpu(), o["row_loss"], w * a * rel + 1e-7, "row_loss")
    _near(out["totals"].cpu(), o["totals"], (w * (a + 1) * rel).sum() + 1e-6, "totals")
    if out["grad"] is None:
        return
    got = out["grad"].cpu().numpy()
    assert np.all(got[len(s):] == 7.0)                     # rows past the images
    for i in range(len(k)):
        lo, hi = int(cu[i]), int(cu[i + 1])
        tol = w[i] * a[i] * (rel[i] + 4 * LOGP * size) * (1 + np.abs(o["grad"][lo:hi]) /
                                                          (w[i] * a[i] + 1e-9))
        _near(got[lo:hi], o["grad"][lo:hi], tol + 1e-7, f"grad {i}")
        if hi > lo:
            assert got[lo] == 0


@pytest.mark.parametrize("std", [0.5, 3.0, 40.0])
def test_pl_policy_loss_matches_oracle(std):
    lens = [1, 2, 2, 9, 33, 34, 197, 65, 258, 300, 0, 513, 577, 1500, 2049]
    k = [0, 0, 1, 8, 32, 1, 60, 64, 257, 0, 0, 511, 130, 900, 2048]
    q = _sequences(lens, k, std, int(std))
    out, st = _run_sequences(q)
    assert st == 0
    _check_sequences(q, out)


def test_pl_policy_loss_options_same_bits_and_weights():
    rng = np.random.default_rng(4)
    lens = rng.integers(20, 198, 1300)
    k = np.minimum(rng.integers(0, 25, 1300), lens - 5)
    q = _sequences(list(lens), list(k), 1.5, 5)
    a, st = _run_sequences(q)
    b, _ = _run_sequences(q, stream=torch.cuda.Stream())
    assert st == 0
    for n in a:
        assert torch.equal(a[n], b[n])
    _check_sequences(q, a)
    c, _ = _run_sequences(q, grad=False)
    assert torch.equal(a["totals"], c["totals"]) and torch.equal(a["logp"], c["logp"])
    c, _ = _run_sequences(q, weights=False, ref=False)
    _check_sequences(q, c, weights=False, ref=False)
    q[7][::3] = 0.0                                        # weight 0: no part
    c, _ = _run_sequences(q)
    assert not c["logp"][::3].any() and not c["row_loss"][::3].any()
    q[2][::3] = 0
    _check_sequences(q, c)


def test_pl_policy_loss_agrees_with_the_logprob_entry():
    lens, k = [197] * 40, list(range(1, 41))
    q = _sequences(lens, k, 1.0, 8)
    s, cu, kk, order, old, adv, rf, w = q
    out, _ = _run_sequences(q, ref=False, weights=False)
    logp, grad = torch.zeros(40, device=dev()), torch.zeros(len(s), device=dev())
    ratio = np.exp(O.pl_policy_loss(s, cu, kk, order, old, adv)["logp"] - old)
    clipped = ratio * adv > np.clip(ratio, .8, 1.2) * adv
    P.dora_pl_logprob(f32(s), i32(cu), i32(kk), i32(order), logp, grad=grad,
                      dlogp=f32(np.where(clipped, 0, -ratio * adv)))
    assert np.allclose(logp.cpu(), out["logp"].cpu(), rtol=1e-5)
    assert np.allclose(grad.cpu(), out["grad"][:len(s)].cpu(), rtol=1e-3, atol=1e-4)


@pytest.mark.parametrize("value", [-np.inf, float(np.finfo(np.float32).min)])
def test_pl_policy_loss_tokens_of_probability_zero(value):
    """Tokens that are never removed because their score is -inf, or fp32's lowest
    value, are as good as absent; more of them than threads."""
    q = _sequences([7, 42, 173, 902], [2, 30, 130, 900], 1.5, 14)
    s, cu, k, order = q[:4]
    rng = np.random.default_rng(15)
    scores, places, moved = [], [], np.full_like(order, -1)
    for i in range(len(k)):
        n = int(cu[i + 1] - cu[i]) - 1
        at = np.sort(rng.permutation(n + 300)[:n])         # of the image's own tokens
        img = np.full(n + 300, value, dtype=np.float32)
        img[at] = s[cu[i] + 1:cu[i + 1]]
        moved[i, :k[i]] = at[order[i, :k[i]]]
        start = sum(len(x) for x in scores)
        places.append(np.concatenate([[start], start + 1 + at]))
        scores.append(np.concatenate([[0.0], img]).astype(np.float32))
    cu2 = O.cu_from_counts([len(x) for x in scores])
    out, st = _run_sequences((np.concatenate(scores), cu2, k, moved) + q[4:])
    assert st == 0
    places = torch.from_numpy(np.concatenate(places)).to(dev())
    rest = torch.ones(int(cu2[-1]), dtype=torch.bool, device=dev())
    rest[places] = False
    assert not out["grad"][:int(cu2[-1])][rest].any()
    out["grad"] = torch.cat([out["grad"][places], out["grad"][-5:]])
    _check_sequences(q, out)


def test_pl_policy_loss_removed_token_of_probability_zero():
    s = np.array([0, .5, -np.inf, 1., 0, .5, -.5, 1.], dtype=np.float32)
    cu, k = np.array([0, 4, 8]), np.array([2, 2])
    order = np.array([[1, 0], [1, 0]])                     # log-probability -inf; finite
    one, lp = np.ones(2, dtype=np.float32), O.pl_logprob(s[5:], [1, 0])
    out, st = _run_sequences((s, cu, k, order, np.float32([-1, lp]), one, one, one), ref=False)
    assert st == 0 and float(out["logp"][0]) == -np.inf
    assert float(out["row_loss"][0]) == 0 and not out["grad"][:4].any()
    assert abs(float(out["logp"][1]) - lp) < 1e-6 and abs(float(out["totals"][0]) + 1) < 1e-5


def test_policy_loss_totals_of_an_infinite_loss():
    """A ratio past fp32's range with A < 0 is a loss of +inf, and so is the total."""
    rows = 3000
    c = _Case(rows, 8, F32, 16)
    c.old[7], c.adv[7], c.w[7] = -300.0, -1.0, 1.0
    if c.actions[7] < 0:
        c.actions[7] = 0
    out = c.run()
    assert float(out["row_loss"][7]) == np.inf and float(out["totals"][0]) == np.inf
    assert float(out["totals"][1]) == np.inf and bool(torch.isfinite(out["totals"][2:]).all())


def test_pl_policy_loss_device_errors():
    q = _sequences([6, 6, 6, 6], [2, 2, 2, 2], 1.0, 9)
    q[3][1] = [0, 0]                                       # repeated
    q[3][2] = [1, 7]                                       # out of range
    out, st = _run_sequences(q)
    assert st == O.DORA_ERR_DEVICE_BAD_COUNT
    lp = out["logp"].cpu().numpy()
    assert np.isnan(lp).tolist() == [False, True, True, False]
    g = out["grad"].cpu().numpy()
    assert np.isnan(g[6:18]).all() and np.isfinite(g[:6]).all() and np.isfinite(g[18:24]).all()
    q = _sequences([6, 6], [2, 2], 1.0, 10)
    q[2][1] = 3                                            # k above k_cap: clamped
    out, st = _run_sequences(q)
    assert st == O.DORA_ERR_DEVICE_BAD_COUNT and bool(torch.isfinite(out["logp"]).all())
    q = _sequences([2051, 5], [3, 2], 1.0, 11)             # longer than 2048 visual tokens
    out, st = _run_sequences(q)
    assert st == O.DORA_ERR_DEVICE_SEQLEN and float(out["logp"][0]) == 0
    assert not out["grad"][:2051].any()
    tot = torch.full((6,), 3.0, device=dev())
    e, ei = torch.zeros(0, device=dev()), torch.zeros(0, dtype=torch.int32, device=dev())
    P.dora_pl_policy_loss(torch.zeros(4, device=dev()), i32([0]), ei,
                          torch.zeros(0, 3, dtype=torch.int32, device=dev()), e, e, e,
                          P.alloc_policy_workspace(dev()), totals=tot)
    assert not tot.any()
