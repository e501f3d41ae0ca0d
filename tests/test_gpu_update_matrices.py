"""The rollout's record, a loss of the caller's own and the step that updates matrices, run
together as a training program would: log-probabilities -> loss -> gradients -> norm ->
Muon on the matrices, Adam on the vectors; eagerly, captured, and in the example."""
import numpy as np
import pytest
import torch

import __graft_entry__ as G
import oracle as O
import paper_2609_34325_gb300 as P
from helpers import dev
from paper_2609_34325_gb300 import update as U

pytestmark = pytest.mark.gpu

F32, BF16, I32 = torch.float32, torch.bfloat16, torch.int32


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    G.build()
    P.load_library()
    torch.cuda.set_device(0)


def _np(t):
    return t.detach().double().cpu().numpy()


class _Policy:
    """Two linear layers and a bias in fp32, their moments and gradients."""

    def __init__(self, features=96, hidden=160, tokens=300, rows=64, seed=1):
        g = torch.Generator(device=dev()).manual_seed(seed)

        def randn(*s):
            return torch.randn(*s, generator=g, device=dev())

        self.x = randn(rows, features)
        self.p = [randn(hidden, features) * 0.1, randn(tokens, hidden) * 0.1, randn(tokens) * 0.1]
        self.g = [torch.zeros_like(t) for t in self.p]
        self.m = [torch.zeros_like(t) for t in self.p]
        self.v = torch.zeros_like(self.p[2])
        self.copies = [t.to(BF16) for t in self.p]
        self.tokens = torch.randint(0, tokens, (rows,), generator=g, device=dev(), dtype=I32)
        self.tokens[3] = -1
        self.dlogp = randn(rows) / rows
        self.dentropy = torch.full((rows,), -0.01 / rows, device=dev())
        self.logits = torch.zeros(rows, tokens, device=dev())
        self.logp, self.entropy = torch.zeros(rows, device=dev()), torch.zeros(rows, device=dev())
        self.stats, self.norm = torch.zeros(rows, 2, device=dev()), torch.zeros(2, device=dev())
        self.all = P.ParamList(self.g)
        self.matrices = P.MatrixList(self.g[:2], params=self.p[:2], momentum=self.m[:2],
                                     copies=self.copies[:2])
        self.vectors = P.ParamList(self.g[2:], params=self.p[2:], exp_avg=self.m[2:],
                                   exp_avg_sq=[self.v], copies=self.copies[2:])
        self.state = P.alloc_adam_state(dev())

    def step(self):
        h = torch.relu(self.x @ self.p[0].t())
        torch.addmm(self.p[2], h, self.p[1].t(), out=self.logits)
        P.dora_token_logprob(self.logits, self.tokens, self.logp, entropy=self.entropy,
                             norm=self.stats)
        P.dora_token_logprob_grad(self.logits, self.tokens, self.stats, self.logits,
                                  dlogp=self.dlogp, dentropy=self.dentropy, entropy=self.entropy)
        torch.mm(self.logits.t(), h, out=self.g[1])
        torch.sum(self.logits, 0, out=self.g[2])
        torch.mm(((self.logits @ self.p[1]) * (h > 0)).t(), self.x, out=self.g[0])
        P.dora_grad_norm(self.all, 0.02, self.norm)
        P.dora_muon_step(self.matrices, 1e-2, momentum=0.9, weight_decay=0.1, clip=self.norm)
        P.dora_adam_step(self.vectors, self.state, 1e-2, clip=self.norm)


def test_one_step_matches_the_oracle():
    a = _Policy()
    x, p = _np(a.x), [_np(t) for t in a.p]
    tokens = a.tokens.cpu().numpy()
    a.step()
    torch.cuda.synchronize()
    h = np.maximum(x @ p[0].T, 0)
    z = h @ p[1].T + p[2]
    f = O.token_logprob(z, tokens)
    # logits are two fp32 products of 96 and 160 terms: 1e-5 of values up to 10
    assert np.allclose(_np(a.logp), f["logp"], atol=2e-4)
    assert np.allclose(_np(a.entropy), f["entropy"], atol=2e-4)
    assert a.logp[3] == 0 and not f["logp"][3]
    dz = O.token_logprob_grad(z, tokens, _np(a.dlogp), _np(a.dentropy))
    want = [((dz @ p[1]) * (h > 0)).T @ x, dz.T @ h, dz.sum(0)]
    for g, w in zip(a.g, want):
        assert np.linalg.norm(_np(g) - w) <= 1e-4 * np.linalg.norm(w)
    norm, factor = O.grad_norm(want, 0.02)
    assert factor < 1 and abs(float(a.norm[0]) - norm) <= 1e-4 * norm
    for i in range(2):
        rows, cols = p[i].shape
        pr, mr = O.muon_step(p[i], 0 * p[i], want[i], 1e-2, 0.9, True, 0.1,
                             max(1, rows / cols) ** 0.5, 5, factor)
        assert np.linalg.norm(_np(a.m[i]) - mr) <= 1e-3 * np.linalg.norm(mr)
        # the iteration's own bound, and what it makes of gradients that are 1e-4 off: directions
        # below a hundredth of the norm are raised by up to 3.4445^5 = 485 (a low-rank
        # gradient's small ones carry less than a tenth of the update)
        moved = np.linalg.norm(pr - p[i] * (1 - 1e-3))
        assert np.linalg.norm(_np(a.p[i]) - pr) <= 2e-2 * moved
        assert torch.equal(a.copies[i], a.p[i].to(BF16))
    pr, _, _ = O.adam_step(p[2], 0 * p[2], 0 * p[2], want[2], 1, 1e-2, 0.9, 0.999, 1e-8, 0.0,
                           factor)
    big = np.abs(want[2]) > 1e-2 * np.abs(want[2]).max()    # Adam's first step is the sign
    assert np.allclose(_np(a.p[2])[big], pr[big], atol=1e-4)


def test_gradients_are_the_loss_differences():
    a = _Policy(features=20, hidden=24, tokens=40, rows=6, seed=3)
    p0 = [t.clone() for t in a.p]

    def loss(which, where, by):
        x, w = _np(a.x), [_np(t).copy() for t in p0]
        w[which][where] += by
        z = np.maximum(x @ w[0].T, 0) @ w[1].T + w[2]
        f = O.token_logprob(z, a.tokens.cpu().numpy())
        return (_np(a.dlogp) * f["logp"] + _np(a.dentropy) * f["entropy"]).sum()

    a.step()
    for which, where in ((0, (3, 5)), (0, (20, 19)), (1, (7, 2)), (1, (39, 23)), (2, (4,))):
        slope = (loss(which, where, 1e-5) - loss(which, where, -1e-5)) / 2e-5
        assert abs(float(a.g[which][where]) - slope) <= 1e-5 + 1e-3 * abs(slope)


def test_steps_eager_and_captured():
    eager, captured = _Policy(seed=5), _Policy(seed=5)
    warm = _Policy(seed=6)                     # the libraries' own set-up
    warm.step()
    for _ in range(3):
        eager.step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        warm.step()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            captured.step()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    # torch's own products may take other kernels on another stream: near, not equal
    for x, y in zip(eager.p + eager.m, captured.p + captured.m):
        assert torch.allclose(x, y, rtol=0, atol=1e-3 * float(x.abs().max()))
    assert int(captured.state[:8].view(torch.int64)) == 3


def test_two_lists_on_two_streams():
    # their own memory each: calls may overlap
    one, two = [_Policy(seed=7) for _ in range(2)]
    ref = _Policy(seed=7)
    for a in (one, two, ref):
        for i, g in enumerate(a.g):
            g.copy_(torch.randn(g.shape, generator=torch.Generator(device=dev()).manual_seed(i),
                                device=dev()))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(4):
        for a, s in zip((one, two), streams):
            P.dora_muon_step(a.matrices, 1e-2, stream=s)
        P.dora_muon_step(ref.matrices, 1e-2)
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(one.p[i], ref.p[i]) and torch.equal(two.p[i], ref.p[i])


def test_the_example_takes_down_what_the_policy_was():
    heads = U.HeadUpdate(64, 20, dev(), seed=3, epochs=1, muon=True)
    task = U.RemovalTask(24, 44, 64, dev(), seed=4)
    r = heads.act(*task.batch())
    logits, _ = heads.forward(r.z_cls, r.z_tok)
    f = O.token_logprob(_np(logits), r.budgets.cpu().numpy(), r.legal.cpu().numpy(),
                        top=U.ALTERNATIVES)
    assert np.allclose(_np(r.budget_logp), f["logp"], atol=1e-5)
    assert np.allclose(_np(r.entropy), f["entropy"], atol=1e-5)
    assert np.array_equal(r.top_budgets.cpu().numpy(), f["top_tokens"])
    # and the step: the matrix by Muon, the vectors by Adam, on gradients clipped together
    before = [_np(w) for w in heads.weights]
    reward, lost = task.rewards(r)
    heads.update(r, U.normalised(reward), U.normalised(-lost))
    torch.cuda.synchronize()
    norm, factor = O.grad_norm([_np(g) for g in heads.grads], heads.max_norm)
    pr, _ = O.muon_step(before[0], 0 * before[0], _np(heads.grads[0]), heads.lr, 0.95, True, 0.0,
                        0.2 * 64 ** 0.5, 5, factor)
    moved = np.linalg.norm(pr - before[0])
    assert moved > 0 and np.linalg.norm(_np(heads.weights[0]) - pr) <= 6e-3 * moved + 1e-6
    for w, p, g in zip(heads.weights[1:], before[1:], heads.grads[1:]):
        want, _, _ = O.adam_step(p, 0 * p, 0 * p, _np(g), 1, heads.lr, 0.9, 0.999, 1e-8, 0.0,
                                 factor)
        assert np.all(np.abs(_np(w) - want) <= 1e-5 * heads.lr * 10 + 2.0 ** -22 * np.abs(want))
    for w, c in zip(heads.weights, heads.copies):
        assert torch.equal(c, w.to(BF16))
    assert int(heads.status.item()) == 0


def test_the_example_runs_with_muon():
    h = U.main(["--updates", "4", "--images", "32", "--tokens", "44", "--features", "64",
                "--muon"])
    assert h.shape == (4, 5) and bool(torch.isfinite(h).all())
