"""The policy update of the actor's two heads, from a rollout's actions to
changed weights (App. D.2: clipped PPO, a few epochs a rollout; Table 4: Adam).

    python -m paper_2609_34325_gb300.update [--updates 60] [--images 256] [--tokens 196] [--muon]

``HeadUpdate`` holds a linear budget head and a linear selector on the
encoder's features (Z_CLS [B, f] and the tokens' Z [T, f] of a packed batch):
fp32 master weights, their Adam moments and the bf16 copies that the forward
reads.  ``act`` samples a budget and an ordered removal sequence for every
image, with their log-probabilities, the budgets' entropies and what else they
could have been (dora_token_logprob); ``update`` runs the epochs: forward of the
heads, the clipped losses with their gradients (dora_policy_loss,
dora_pl_policy_loss), the weights' gradients, their global norm (dora_grad_norm)
and an Adam step on the clipped gradients (dora_adam_step), or, with ``muon``, a
Muon step on the budget head's matrix (dora_muon_step) and Adam on the vectors.
Nothing in it waits for the device.

Run as a command it learns a synthetic task (random features, a hidden
importance of every token; an action is worth the tokens it removes less the
importance it loses) and prints how the reward rises.
"""
from __future__ import annotations

import argparse

import torch

from . import (MatrixList, ParamList, alloc_adam_state, alloc_policy_workspace, dora_adam_step,
               dora_grad_norm, dora_muon_step, dora_pl_policy_loss, dora_pl_sample,
               dora_policy_loss, dora_token_logprob)

_BF16, _F32, _I32 = torch.bfloat16, torch.float32, torch.int32


def _gumbel(shape, generator, device):
    u = torch.rand(shape, generator=generator, device=device).clamp_(min=1e-9)
    return -(-u.log()).log()


class Rollout:
    """What a rollout leaves for its update: features, boundaries, the actions
    taken and their log-probabilities when they were taken; the budgets' entropies,
    and the most probable budgets [B, ALTERNATIVES] with their log-probabilities."""

    def __init__(self, z_cls, z_tok, cu, budgets, legal, k, order, budget_logp, order_logp,
                 entropy=None, top_budgets=None, top_logp=None):
        self.z_cls, self.z_tok, self.cu = z_cls, z_tok, cu
        self.budgets, self.legal, self.k, self.order = budgets, legal, k, order
        self.budget_logp, self.order_logp = budget_logp, order_logp
        self.entropy, self.top_budgets, self.top_logp = entropy, top_budgets, top_logp


ALTERNATIVES = 3


class HeadUpdate:
    """A budget head over the counts 2, 4, ..., 2 * budgets and a selector, with
    their update.  An image of n visual tokens may lose n - 4 at most
    (App. A.2), so its first (n - 4) // 2 counts are legal."""

    def __init__(self, features: int, budgets: int, device, seed: int = 0, lr: float = 1e-2,
                 clip: float = 0.2, entropy_coef: float = 0.01, max_norm: float = 0.5,
                 epochs: int = 3, muon: bool = False):
        g = torch.Generator(device=device).manual_seed(seed)
        self.features, self.budgets = features, budgets
        self.lr, self.clip, self.entropy_coef = lr, clip, entropy_coef
        self.max_norm, self.epochs = max_norm, epochs
        shapes = ((budgets, features), (budgets,), (features,))
        self.weights = [torch.randn(s, generator=g, device=device) * 0.02 for s in shapes]
        self.copies = [w.to(_BF16) for w in self.weights]
        self.grads = [torch.zeros(s, device=device) for s in shapes]
        self.moments = [[torch.zeros(s, device=device) for s in shapes] for _ in range(2)]
        self.list = ParamList(self.grads, params=self.weights, exp_avg=self.moments[0],
                              exp_avg_sq=self.moments[1], copies=self.copies)
        # Muon for the matrix, then Adam for the vectors alone; the norm is over all of them
        self.matrices, self.adam_list = None, self.list
        if muon:
            self.matrices = MatrixList(self.grads[:1], params=self.weights[:1],
                                       momentum=self.moments[0][:1], copies=self.copies[:1],
                                       scales=[0.2 * max(shapes[0]) ** 0.5])
            self.adam_list = ParamList(self.grads[1:], params=self.weights[1:],
                                       exp_avg=self.moments[0][1:], exp_avg_sq=self.moments[1][1:],
                                       copies=self.copies[1:])
        self.adam = alloc_adam_state(device)
        self.norm = torch.zeros(2, device=device)
        self.workspace = alloc_policy_workspace(device)
        self.totals = torch.zeros(2, 6, device=device)
        self.status = torch.zeros(1, dtype=_I32, device=device)
        self.generator = g

    def forward(self, z_cls, z_tok):
        """Budget logits bf16 [B, budgets] and selector scores fp32 [T]."""
        w, b, s = self.copies
        return torch.addmm(b, z_cls, w.t()), (z_tok @ s).float()

    def act(self, z_cls, z_tok, cu) -> Rollout:
        """Samples every image's budget and removal order (bf16 features, cu
        int32 [B + 1]) and takes down their log-probabilities."""
        logits, scores = self.forward(z_cls, z_tok)
        batch, dev = z_cls.shape[0], z_cls.device
        n = cu[1:] - cu[:-1] - 1
        legal = ((n - 4) // 2).clamp(0, self.budgets).to(_I32)
        noisy = logits.float() + _gumbel(logits.shape, self.generator, dev)
        noisy.masked_fill_(torch.arange(self.budgets, device=dev) >= legal[:, None], -torch.inf)
        budgets = torch.where(legal > 0, noisy.argmax(1), -1).to(_I32)
        k = (2 * (budgets + 1)).to(_I32)
        order = torch.empty(batch, 2 * self.budgets, dtype=_I32, device=dev)
        dora_pl_sample(scores, _gumbel(scores.shape, self.generator, dev), cu, k, order,
                       status=self.status)
        none = torch.zeros(batch, device=dev)
        budget_logp, order_logp = torch.empty(batch, device=dev), torch.empty(batch, device=dev)
        entropy = torch.empty(batch, device=dev)
        top_logp = torch.empty(batch, ALTERNATIVES, device=dev)
        top_budgets = torch.empty(batch, ALTERNATIVES, dtype=_I32, device=dev)
        dora_token_logprob(logits, budgets, budget_logp, legal=legal, entropy=entropy,
                           top_logp=top_logp, top_tokens=top_budgets, status=self.status)
        dora_pl_policy_loss(scores, cu, k, order, none, none, order_logp, status=self.status)
        return Rollout(z_cls, z_tok, cu, budgets, legal, k, order, budget_logp, order_logp,
                       entropy, top_budgets, top_logp)

    def losses(self, r: Rollout, budget_adv, order_adv):
        """One forward and backward of both heads: ``grads`` of the weights from
        the mean clipped losses, whose terms are left in ``totals``."""
        logits, scores = self.forward(r.z_cls, r.z_tok)
        batch = logits.shape[0]
        share = torch.full((batch,), 1.0 / batch, device=logits.device)
        logp = torch.empty_like(share)
        # rows past the images are not written: their scores have no gradient
        dlogits, dscores = torch.empty_like(logits), torch.zeros_like(scores)
        dora_policy_loss(logits, r.budgets, r.budget_logp, budget_adv, logp, self.workspace,
                         grad=dlogits, legal=r.legal, weights=share, clip_low=self.clip,
                         clip_high=self.clip, entropy_coef=self.entropy_coef,
                         totals=self.totals[0], status=self.status)
        dora_pl_policy_loss(scores, r.cu, r.k, r.order, r.order_logp, order_adv, logp,
                            self.workspace, grad=dscores, weights=share, clip_low=self.clip,
                            clip_high=self.clip, totals=self.totals[1], status=self.status)
        dw, db, ds = self.grads
        dw.copy_(dlogits.t() @ r.z_cls)
        db.copy_(dlogits.float().sum(0))
        ds.copy_(dscores @ r.z_tok.float())

    def update(self, r: Rollout, budget_adv, order_adv):
        """The epochs of one rollout, on advantages normalised for each head."""
        for _ in range(self.epochs):
            self.losses(r, budget_adv, order_adv)
            dora_grad_norm(self.list, self.max_norm, self.norm)
            if self.matrices is not None:
                dora_muon_step(self.matrices, self.lr, clip=self.norm, status=self.status)
            dora_adam_step(self.adam_list, self.adam, self.lr, clip=self.norm)


def normalised(x):
    return (x - x.mean()) / (x.std() + 1e-6)


class RemovalTask:
    """A synthetic task: tokens of random features whose importance a hidden
    direction gives; an image's reward is the share of its tokens removed less
    `price` times the importance lost with them."""

    def __init__(self, images: int, tokens: int, features: int, device, seed: int = 1,
                 price: float = 2.0):
        self.g = torch.Generator(device=device).manual_seed(seed)
        self.images, self.tokens, self.features, self.price = images, tokens, features, price
        self.device = device
        self.direction = torch.randn(features, generator=self.g, device=device) / features ** 0.5

    def batch(self):
        n = torch.randint(self.tokens // 2, self.tokens + 1, (self.images,), generator=self.g,
                          device=self.device)
        cu = torch.zeros(self.images + 1, dtype=_I32, device=self.device)
        cu[1:] = (n + 1).cumsum(0)
        rows = self.images * (self.tokens + 1)   # a capacity: the live rows are cu[-1]
        z = torch.randn(rows, self.features, generator=self.g, device=self.device).to(_BF16)
        return z[cu[:-1].long()], z, cu

    def rewards(self, r: Rollout):
        """(rewards [B], importance of the removed tokens [B])."""
        importance = torch.sigmoid(4 * (r.z_tok.float() @ self.direction))
        taken = r.order >= 0
        at = r.cu[:-1, None].long() + 1 + r.order.clamp(min=0).long()
        lost = torch.where(taken, importance[at], 0.0).sum(1)
        n = (r.cu[1:] - r.cu[:-1] - 1).clamp(min=1)
        k = taken.sum(1)
        return (k - self.price * lost) / n, lost / k.clamp(min=1)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--updates", type=int, default=60)
    ap.add_argument("--images", type=int, default=256)
    ap.add_argument("--tokens", type=int, default=196)
    ap.add_argument("--features", type=int, default=128)
    ap.add_argument("--seed", type=int, default=0)
    ap.add_argument("--muon", action="store_true", help="Muon for the budget head's matrix")
    a = ap.parse_args(argv)
    dev = torch.device("cuda:0")
    torch.cuda.set_device(dev)
    heads = HeadUpdate(a.features, (a.tokens - 4) // 2, dev, seed=a.seed, muon=a.muon)
    task = RemovalTask(a.images, a.tokens, a.features, dev, seed=a.seed + 1)
    history = []
    for u in range(a.updates):
        r = heads.act(*task.batch())
        reward, lost = task.rewards(r)
        heads.update(r, normalised(reward), normalised(-lost))
        history.append(torch.stack([reward.mean(), lost.mean(), heads.norm[0],
                                    heads.totals[0, 4], heads.totals[0, 3]]))
        if u % 10 == 9 or u == 0:
            v = history[-1].tolist()
            print(f"update {u + 1:3d}: reward {v[0]:+.4f}  importance of removed tokens "
                  f"{v[1]:.3f}  gradient norm {v[2]:.3f}  clipped {v[3]:.2f}  entropy {v[4]:.2f}")
    if int(heads.status.item()):
        raise RuntimeError(f"device status {int(heads.status.item())}")
    return torch.stack(history)


if __name__ == "__main__":
    main()
