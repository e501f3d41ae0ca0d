"""The operators of one policy update, as cases that can be timed and compared.

Five kinds, in the order in which an update calls them:

* ``policy``    clipped policy loss with KL and entropy terms of categorical actions, logits to
                their gradient;
* ``sequence``  the same loss of ordered removal sequences (Plackett-Luce), scores to their
                gradient;
* ``norm``      the global gradient norm over many tensors;
* ``clip``      the gradients scaled to a largest norm, into buffers of their own;
* ``adam``      an Adam step on many tensors whose gradients are clipped on the way.

``own`` says which form ``run`` computes: false, elementary torch operations in 32 bits; true,
this package's kernels.  Tensors of one type are views of one flat buffer, as a training program
that saves or exchanges them in one piece lays them out, each at a multiple of ``align`` elements.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
F32, F64, I32 = torch.float32, torch.float64, torch.int32
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
BETA1, BETA2, ADAM_EPS = 0.9, 0.999, 1e-8
STEPS_DONE = 100          # Adam steps before the timed ones: moments are filled
MAX_POLICY = 4095 * 50001  # logits of the largest listed loss
MAX_PARAMS = 86_000_000   # elements of the largest listed tensor lists, about


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def _policy(name, rows, classes, dtype, pitch, legal, idle, kl, entropy):
    return {"name": name, "kind": "policy", "rows": rows, "classes": classes, "dtype": dtype,
            "pitch": pitch, "legal": legal, "idle": idle, "kl": kl, "entropy": entropy}


def listed():
    return [
        # the budget head over one rollout batch: 96 counts, feasible ones first, a third of the
        # gates closed; a few microseconds of work
        _policy("policy_budget_256", 256, 96, "float32", 96, True, 0.3, 0.0, 0.01),
        # a token policy's step with padding and a reference policy
        _policy("policy_tokens_2k", 2048, 32000, "bfloat16", 32000, False, 0.15, 0.05, 0.0),
        # the largest: an odd number of classes, so that rows start at any alignment
        _policy("policy_odd_4k", 4095, 50001, "float16", 50001, False, 0.05, 0.02, 0.001),
        # few rows, each long: the rows alone do not fill the card
        _policy("policy_long_8", 8, 131072, "float32", 131072, False, 0.0, 0.05, 0.01),
        # the selector's removals at the first pruning block of a rollout batch
        {"name": "sequence_256", "kind": "sequence", "images": 256, "tokens": 197, "removed": 60,
         "std": 1.0, "idle": 0.25, "kl": 0.0},
        # the 384-pixel backbone, four rollout batches in one update
        {"name": "sequence_384px_1k", "kind": "sequence", "images": 1024, "tokens": 577,
         "removed": 120, "std": 2.0, "idle": 0.1, "kl": 0.05},
        # the actor's gradients: 32 small tensors, latency
        {"name": "norm_actor", "kind": "norm", "layout": "actor", "dim": 768, "depth": 12,
         "count": 0, "elements": 0, "shape_seed": 0, "dtype": "float32", "align": 64},
        # a backbone of base size in mixed types: matrices bf16, vectors fp32
        {"name": "norm_base", "kind": "norm", "layout": "vit", "dim": 768, "depth": 12,
         "count": 0, "elements": 0, "shape_seed": 0, "dtype": "mixed", "align": 64},
        {"name": "clip_actor", "kind": "clip", "layout": "actor", "dim": 768, "depth": 12,
         "count": 0, "elements": 0, "shape_seed": 0, "dtype": "float32", "align": 64,
         "active": True},
        {"name": "clip_base", "kind": "clip", "layout": "vit", "dim": 768, "depth": 12,
         "count": 0, "elements": 0, "shape_seed": 0, "dtype": "float32", "align": 64,
         "active": True},
        # the actor's step: fp32 masters, bf16 copies for the next rollout
        {"name": "adam_actor", "kind": "adam", "layout": "actor", "dim": 768, "depth": 12,
         "count": 0, "elements": 0, "shape_seed": 0, "dtype": "float32", "align": 64,
         "param": "float32", "copy": True, "decay": 0.0},
        # a whole backbone of base size with bf16 gradients
        {"name": "adam_base", "kind": "adam", "layout": "vit", "dim": 768, "depth": 12,
         "count": 0, "elements": 0, "shape_seed": 0, "dtype": "bfloat16", "align": 64,
         "param": "float32", "copy": True, "decay": 0.05},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["policy", "policy", "sequence", "norm", "clip", "adam"])
    if kind == "policy":
        dtype = rng.choice(["float32", "bfloat16", "float16"])
        classes = _log_int(rng, 2, 131072)
        most = MAX_POLICY // classes // (2 if dtype == "float32" else 1)
        rows = _log_int(rng, 1, max(1, min(65536, most)))
        return {"kind": kind, "rows": rows, "classes": classes, "dtype": dtype,
                "pitch": classes + rng.choice([0, 0, 1, 7, -classes % 64]),
                "legal": rng.random() < 0.3, "idle": rng.choice([0.0, 0.1, 0.4]),
                "kl": rng.choice([0.0, 0.05]), "entropy": rng.choice([0.0, 0.01])}
    if kind == "sequence":
        tokens = _log_int(rng, 8, 2049)
        return {"kind": kind, "images": _log_int(rng, 1, min(1024, 600000 // tokens)),
                "tokens": tokens, "removed": min(128, _log_int(rng, 1, tokens - 5)),
                "std": rng.choice([0.5, 1.0, 2.0]), "idle": rng.choice([0.0, 0.25]),
                "kl": rng.choice([0.0, 0.05])}
    case = {"kind": kind, "layout": rng.choice(["actor", "vit", "ragged", "ragged"]),
            "dim": rng.choice([192, 384, 768]), "depth": 12, "count": _log_int(rng, 1, 400),
            "elements": _log_int(rng, 500, MAX_PARAMS // 2), "shape_seed": rng.randrange(1 << 20),
            "dtype": rng.choice(["float32", "bfloat16", "float16", "mixed"]),
            "align": rng.choice([64, 64, 1])}
    if kind == "clip":
        case["active"] = rng.random() < 0.7
    if kind == "adam":
        case["dtype"] = rng.choice(["float32", "bfloat16", "float16"])
        case["param"] = rng.choice(["float32", "float32", "bfloat16"])
        case["copy"] = case["param"] == "float32" and rng.random() < 0.5
        case["decay"] = rng.choice([0.0, 0.05])
    return case


# ---------------------------------------------------------------------------
# tensor lists
# ---------------------------------------------------------------------------

def _shapes(case):
    d, depth = case["dim"], case["depth"]
    if case["layout"] == "actor":  # the deployment actor of a backbone of width d, 196 patches
        return [(64, d + 19), (64,), (1, 64), (1,), (depth, 16), (128, d), (128,), (depth, 128),
                (128, 3), (128,), (128,), (384, 128), (384,), (128, 128), (128,), (128,), (128,),
                (256, 128), (256,), (128, 256), (128,), (128,), (128,), (128, 128), (128,),
                (96, 128), (96,), (128,), (64, 128), (64,), (1, 64), (1,)]
    if case["layout"] == "vit":    # patch embedding, blocks, classifier
        block = [(d,), (d,), (3 * d, d), (3 * d,), (d, d), (d,), (d,), (d,), (4 * d, d), (4 * d,),
                 (d, 4 * d), (d,)]
        return [(d, 768), (d,), (d,), (197, d)] + block * depth + [(d,), (d,), (1000, d), (1000,)]
    rng = random.Random(case["shape_seed"])
    cut = sorted(rng.randint(0, case["elements"]) for _ in range(case["count"] - 1))
    sizes = [b - a for a, b in zip([0] + cut, cut + [case["elements"]])]
    return [(n,) if i % 2 else (1, n) for i, n in enumerate(sizes)]   # empty ones among them


def _groups(case):
    """[(type, elements of the flat buffer, [(offset, shape)])]: one group for each type."""
    by = {}
    for s in _shapes(case):
        name = case["dtype"]
        if name == "mixed":
            name = "bfloat16" if len(s) > 1 else "float32"
        by.setdefault(name, []).append(s)
    out = []
    for name, shapes in by.items():
        at, places = 0, []
        for s in shapes:
            at += -at % case["align"]
            places.append((at, s))
            at += math.prod(s)
        out.append((name, max(1, at), places))
    return out


def _elements(case):
    return [(name, sum(math.prod(s) for _, s in places)) for name, _, places in _groups(case)]


def _views(flat, places):
    return [flat[at:at + math.prod(s)].view(s) for at, s in places]


def _flat(total, places, dtype, make):
    """A flat buffer whose tensors come from `make` and whose gaps are zero."""
    flat = make(total).to(dtype)
    end = 0
    for at, s in places:
        flat[end:at] = 0
        end = at + math.prod(s)
    return flat


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _apart(ratio_log, lo, hi):
    """log ratios whose ratio is not within 0.2% of a clipping bound: there the gradient jumps,
    and the last bit of a log-probability would decide it."""
    for edge in (math.log1p(-lo), math.log1p(hi)):
        ratio_log = torch.where((ratio_log - edge).abs() < 2e-3, ratio_log + 8e-3, ratio_log)
    return ratio_log


def _prepare_policy(case, g):
    rows, v = case["rows"], case["classes"]
    dtype = TYPES[case["dtype"]]
    logits = torch.empty(rows, case["pitch"], dtype=dtype, device=DEV)
    live = rows - int(case["idle"] * rows)
    perm = torch.randperm(rows, generator=g, device=DEV)
    idle = torch.zeros(rows, dtype=torch.bool, device=DEV)
    idle[perm[live:]] = True
    legal = None
    if case["legal"]:   # feasible budgets come first; an idle row may have none
        legal = torch.randint(1, v + 1, (rows,), generator=g, device=DEV, dtype=I32)
        legal = torch.where(idle & (torch.arange(rows, device=DEV) % 2 == 0), 0, legal).to(I32)
    actions = torch.empty(rows, dtype=I32, device=DEV)
    logp = torch.empty(rows, dtype=F64, device=DEV)
    step = max(1, (1 << 25) // case["pitch"])
    for r in range(0, rows, step):
        z = torch.randn(min(step, rows - r), case["pitch"], generator=g, device=DEV) * 2.5
        z = z.to(dtype)
        m = z[:, :v].float()
        if legal is not None:
            out = torch.arange(v, device=DEV) >= legal[r:r + step, None].clamp(min=1)
            m = m.masked_fill(out, -math.inf)
            z[:, :v][out] = math.nan      # what lies past the legal actions is never read
        z[:, v:] = math.nan
        logits[r:r + step] = z
        u = torch.rand(m.shape, generator=g, device=DEV).clamp(min=1e-9)
        a = (m - (-u.log()).log()).argmax(1)
        actions[r:r + step] = a.to(I32)
        logp[r:r + step] = (m.gather(1, a[:, None])[:, 0] - m.logsumexp(1)).double()
    lo, hi = 0.2, 0.2
    delta = _apart(torch.randn(rows, generator=g, device=DEV) * 0.15, lo, hi)
    old = (logp - delta).float()
    ref = (logp + 0.1 * torch.randn(rows, generator=g, device=DEV)).float()
    adv = torch.randn(rows, generator=g, device=DEV)
    # half of the idle rows have no action, the other half no weight
    closed = idle & (torch.arange(rows, device=DEV) % 2 == 0)
    actions[closed] = -1
    # gradients of 16 bits with 5 for the exponent are trained with a scaled loss
    scale = 4096.0 if dtype == torch.float16 else 1.0
    weights = torch.full((rows,), scale / max(1, live), device=DEV)
    weights[idle & ~closed] = 0.0
    return {"logits": logits, "legal": legal, "actions": actions, "old": old,
            "ref": ref if case["kl"] else None, "adv": adv, "weights": weights,
            "lo": lo, "hi": hi}


def _prepare_sequence(case, g):
    b, n0 = case["images"], case["tokens"] - 1
    # lengths between half and all of the tokens, the same for every seed
    n = n0 - torch.arange(b, device=DEV) * 7919 % (n0 - max(1, n0 // 2) + 1)
    cu = torch.zeros(b + 1, dtype=I32, device=DEV)
    cu[1:] = (n + 1).cumsum(0)
    k = (torch.rand(b, generator=g, device=DEV) * (case["removed"] + 1)).long()
    k = torch.minimum(k, n).clamp(min=1)
    perm = torch.randperm(b, generator=g, device=DEV)
    k[perm[b - int(case["idle"] * b):]] = 0           # closed gates
    s = torch.randn(b, n0, generator=g, device=DEV) * case["std"]
    s = s.masked_fill(torch.arange(n0, device=DEV) >= n[:, None], -math.inf)
    u = torch.rand(b, n0, generator=g, device=DEV).clamp(min=1e-9)
    order = (s - (-u.log()).log()).argsort(1, descending=True)[:, :case["removed"]]
    order = order.masked_fill(torch.arange(order.shape[1], device=DEV) >= k[:, None], -1)
    scores = torch.full((int(cu[-1]),), math.nan, device=DEV)   # the CLS rows are not read
    at = cu[:-1, None].long() + 1 + torch.arange(n0, device=DEV)
    inside = torch.arange(n0, device=DEV) < n[:, None]
    scores[at[inside]] = s[inside]
    order = order.to(I32).contiguous()
    logp = _sequence_logp64(s, order, k)
    delta = _apart(torch.randn(b, generator=g, device=DEV) * 0.15, 0.2, 0.2)
    return {"scores": scores, "cu": cu, "k": k.to(I32), "order": order,
            "old": (logp - delta).float(),
            "ref": (logp + 0.1 * torch.randn(b, generator=g, device=DEV)).float()
            if case["kl"] else None,
            "adv": torch.randn(b, generator=g, device=DEV),
            "weights": torch.full((b,), 1.0 / b, device=DEV), "longest": n0, "lo": 0.2, "hi": 0.2}


def _sequence_logp64(s, order, k):
    """log-probabilities of padded score rows (-inf past the tokens), 64 bits."""
    s = s.double()
    taken = order >= 0
    picked = s.gather(1, order.clamp(min=0).long())
    m = s.amax(1, keepdim=True)
    e = (s - m).exp()
    took = torch.where(taken, (picked - m).exp(), 0.0)
    # a token that is removed leaves the rest one by one, from the back: sums without cancellation
    stays = torch.ones_like(e).scatter_add_(1, order.clamp(min=0).long(), -taken.double()) > 0.5
    stays = stays.double() * e
    rest = stays.sum(1, keepdim=True)
    left = rest + took.flip(1).cumsum(1).flip(1)
    return torch.where(taken, picked - m - left.log(), 0.0).sum(1)


def _prepare_list(case, g):
    def randn(scale):
        return lambda n: torch.randn(n, generator=g, device=DEV) * scale

    s = {"case": case, "groups": _groups(case), "grads": []}
    for name, total, places in s["groups"]:
        s["grads"].append(_flat(total, places, TYPES[name], randn(1e-3)))
    s["max_norm"] = 0.5 * 1e-3 * math.sqrt(sum(n for _, n in _elements(case)))
    if case["kind"] == "clip":
        if not case["active"]:
            s["max_norm"] *= 4
        s["clipped"] = [torch.zeros_like(x) for x in s["grads"]]
    if case["kind"] == "adam":
        (_, total, places), = s["groups"]
        s["param"] = _flat(total, places, TYPES[case["param"]], randn(0.02))
        s["m"] = _flat(total, places, F32, randn(3e-4))
        s["v"] = _flat(total, places, F32, lambda n: randn(1e-3)(n).square())
        s["copy"] = s["param"].to(torch.bfloat16) if case["copy"] else None
        s["step"] = STEPS_DONE
        s["lr"] = 3e-4
    s["norm"] = torch.empty(2, device=DEV)
    return s


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    kind = case["kind"]
    if kind == "policy":
        s = _prepare_policy(case, g)
        rows = case["rows"]
        s["grad"] = torch.zeros_like(s["logits"])
    elif kind == "sequence":
        s = _prepare_sequence(case, g)
        rows = case["images"]
        s["grad"] = torch.zeros_like(s["scores"])
    else:
        s = _prepare_list(case, g)
    if kind in ("policy", "sequence"):
        s["logp"], s["row_loss"] = (torch.zeros(rows, device=DEV) for _ in range(2))
        s["entropy"] = torch.zeros(rows, device=DEV)
        s["totals"] = torch.zeros(6, device=DEV)
    s["case"] = case
    if own:   # the handles that a training program makes once
        import paper_2609_34325_gb300 as P
        if kind in ("policy", "sequence"):
            s["workspace"] = P.alloc_policy_workspace(DEV)
        else:
            more = {}
            if kind == "clip":
                more["clipped"] = _all_views(s, s["clipped"])
            if kind == "adam":
                more = {"params": _all_views(s, [s["param"]]), "exp_avg": _all_views(s, [s["m"]]),
                        "exp_avg_sq": _all_views(s, [s["v"]])}
                if s["copy"] is not None:
                    more["copies"] = _all_views(s, [s["copy"]])
                s["adam"] = P.alloc_adam_state(DEV, step=s["step"], beta1=BETA1, beta2=BETA2)
            s["list"] = P.ParamList(_all_views(s, s["grads"]), **more)
    return s


def _all_views(s, flats):
    return [t for (_, _, places), flat in zip(s["groups"], flats) for t in _views(flat, places)]


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    kind = s["case"]["kind"]
    return {"policy": _run_policy, "sequence": _run_sequence, "norm": _run_norm,
            "clip": _run_clip, "adam": _run_adam}[kind](s)


def _row_terms(lp, s, entropy, takes):
    """The loss of each row and its derivative with respect to the log-probability, 32 bits."""
    case = s["case"]
    w, adv = torch.where(takes, s["weights"], 0.0), s["adv"]
    ratio = (lp - s["old"]).exp()
    plain, cut = ratio * adv, ratio.clamp(1 - s["lo"], 1 + s["hi"]) * adv
    inside = plain <= cut
    policy = -torch.minimum(plain, cut)
    g = torch.where(inside, -plain, 0.0)
    kl = torch.zeros_like(lp)
    if s["ref"] is not None:
        x = s["ref"] - lp
        kl = x.expm1() - x
        g = g - case["kl"] * x.expm1()
    row = policy + case["kl"] * kl
    if entropy is not None:
        row = row - case["entropy"] * entropy
    zero = torch.zeros_like(lp)
    row, g = torch.where(takes, w * row, zero), torch.where(takes, w * g, zero)
    terms = torch.stack([
        row, torch.where(takes, w * policy, zero), torch.where(takes, w * kl, zero),
        torch.where(takes, w * entropy, zero) if entropy is not None else zero,
        torch.where(takes & ~inside, w, zero), w])
    return row, g, terms.sum(1)


def _run_policy(s):
    case = s["case"]
    v = case["classes"]
    if own:
        import paper_2609_34325_gb300 as P
        P.dora_policy_loss(s["logits"], s["actions"], s["old"], s["adv"], s["logp"],
                           s["workspace"], grad=s["grad"], classes=v, legal=s["legal"],
                           ref_logp=s["ref"], weights=s["weights"], clip_low=s["lo"],
                           clip_high=s["hi"], kl_coef=case["kl"], entropy_coef=case["entropy"],
                           entropy=s["entropy"], row_loss=s["row_loss"], totals=s["totals"])
        return {"logp": s["logp"], "entropy": s["entropy"], "row_loss": s["row_loss"],
                "totals": s["totals"], "grad": s["grad"][:, :v]}
    takes = (s["actions"] >= 0) & (s["weights"] != 0)
    z = s["logits"][:, :v].float()
    use = takes[:, None]
    if s["legal"] is not None:
        use = use & (torch.arange(v, device=DEV) < s["legal"][:, None])
        z = torch.where(use, z, -math.inf)
        z[:, 0] = torch.where(takes, z[:, 0], 0.0)      # idle rows: any finite row
    else:
        z = torch.where(use, z, 0.0)
    z = z - z.amax(1, keepdim=True)
    e = z.exp()
    total = e.sum(1, keepdim=True)
    logq = z - total.log()
    p = e / total
    a = s["actions"].clamp(min=0).long()[:, None]
    lp = torch.where(takes, logq.gather(1, a)[:, 0], 0.0)
    plogp = torch.where(p > 0, p * logq, 0.0)
    entropy = torch.where(takes, -plogp.sum(1), 0.0)
    row, g, totals = _row_terms(lp, s, entropy, takes)
    grad = -g[:, None] * p
    if case["entropy"]:
        w = torch.where(takes, s["weights"], 0.0) * case["entropy"]
        grad = grad + w[:, None] * (plogp + p * entropy[:, None])
    grad.scatter_add_(1, a, g[:, None])
    grad = torch.where(use, grad, 0.0)
    return {"logp": lp, "entropy": entropy, "row_loss": row, "totals": totals,
            "grad": grad.to(s["logits"].dtype)}


def _run_sequence(s):
    case = s["case"]
    if own:
        import paper_2609_34325_gb300 as P
        P.dora_pl_policy_loss(s["scores"], s["cu"], s["k"], s["order"], s["old"], s["adv"],
                              s["logp"], s["workspace"], grad=s["grad"], ref_logp=s["ref"],
                              weights=s["weights"], clip_low=s["lo"], clip_high=s["hi"],
                              kl_coef=case["kl"], row_loss=s["row_loss"], totals=s["totals"])
        return {"logp": s["logp"], "row_loss": s["row_loss"], "totals": s["totals"],
                "grad": s["grad"]}
    n0, order = s["longest"], s["order"]
    lo, n = s["cu"][:-1].long(), (s["cu"][1:] - s["cu"][:-1] - 1).long()
    k = s["k"].long()
    cols = torch.arange(n0, device=DEV)
    inside = cols < n[:, None]
    at = torch.where(inside, lo[:, None] + 1 + cols, 0)
    z = torch.where(inside, s["scores"][at], -math.inf)
    m = z.amax(1, keepdim=True)
    e = (z - m).exp()
    taken = torch.arange(order.shape[1], device=DEV) < k[:, None]
    pick = torch.where(taken, order, 0).long()
    when = torch.zeros(z.shape, dtype=torch.long, device=DEV).scatter_add_(
        1, pick, torch.where(taken, torch.arange(1, order.shape[1] + 1, device=DEV), 0))
    rest = torch.where(when == 0, e, 0.0).sum(1, keepdim=True)
    left = rest + torch.where(taken, e.gather(1, pick), 0.0).flip(1).cumsum(1).flip(1)
    terms = torch.where(taken, (z - m).gather(1, pick) - left.log(), 0.0)
    takes = (k > 0) & (s["weights"] != 0)
    lp = terms.sum(1)
    # the old log-probability is taken off term by term: the sum of the differences stays small,
    # and with it what 32 bits lose of a ratio of long sequences
    share = torch.where(taken, terms - (s["old"] / k.clamp(min=1))[:, None], 0.0)
    near = dict(s, old=torch.zeros_like(lp))
    if s["ref"] is not None:
        near["ref"] = s["ref"] - s["old"]
    row, g, totals = _row_terms(share.sum(1), near, None, takes)
    inv = torch.where(taken, 1.0 / left, 0.0).cumsum(1)
    last = (k - 1).clamp(min=0)[:, None]
    upto = torch.where(when > 0, inv.gather(1, (when - 1).clamp(min=0)), inv.gather(1, last))
    dl = torch.where(when > 0, 1.0, 0.0) - e * upto
    grad = torch.zeros_like(s["scores"])
    grad[at[inside]] = torch.where(takes[:, None], g[:, None] * dl, 0.0)[inside]
    return {"logp": torch.where(takes, lp, 0.0), "row_loss": row, "totals": totals, "grad": grad}


def _norm_plain(s):
    """[norm, factor] in 32 bits."""
    norm = torch.stack([x.float().square().sum() for x in s["grads"]]).sum().sqrt()
    return norm, torch.clamp(s["max_norm"] / norm, max=1.0)


def _run_norm(s):
    if own:
        import paper_2609_34325_gb300 as P
        P.dora_grad_norm(s["list"], s["max_norm"], s["norm"])
        return s["norm"]
    return torch.stack(_norm_plain(s))


def _run_clip(s):
    if own:
        import paper_2609_34325_gb300 as P
        P.dora_clip_grads(s["list"], s["max_norm"], s["norm"])
        return {"norm": s["norm"], "clipped": s["clipped"]}
    norm, f = _norm_plain(s)
    s["clipped"] = [(x.float() * f).to(x.dtype) for x in s["grads"]]
    return {"norm": torch.stack([norm, f]), "clipped": s["clipped"]}


def _run_adam(s):
    case = s["case"]
    if own:
        import paper_2609_34325_gb300 as P
        P.dora_grad_norm(s["list"], s["max_norm"], s["norm"])
        P.dora_adam_step(s["list"], s["adam"], s["lr"], beta1=BETA1, beta2=BETA2, eps=ADAM_EPS,
                         weight_decay=case["decay"], clip=s["norm"])
        return {k: s[k] for k in ("norm", "param", "m", "v", "copy")}
    norm, f = _norm_plain(s)
    s["step"] += 1
    grad = s["grads"][0].float() * f
    s["m"] = BETA1 * s["m"] + (1 - BETA1) * grad
    s["v"] = BETA2 * s["v"] + (1 - BETA2) * grad.square()
    root = (s["v"] / (1 - BETA2 ** s["step"])).sqrt() + ADAM_EPS
    p = s["param"].float() * (1 - s["lr"] * case["decay"])
    p = p - (s["lr"] / (1 - BETA1 ** s["step"])) * s["m"] / root
    s["param"] = p.to(s["param"].dtype)
    s["copy"] = p.to(torch.bfloat16) if case["copy"] else None
    return {"norm": torch.stack([norm, f]), "param": s["param"], "m": s["m"], "v": s["v"],
            "copy": s["copy"]}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "policy":
        rows, v, size = case["rows"], case["classes"], TYPES[case["dtype"]].itemsize
        live = rows - int(case["idle"] * rows)
        read = v / 2 if case["legal"] else v           # legal counts are spread over 1..v
        rowwise = 4 * rows * (4 + bool(case["legal"]) + bool(case["kl"]) + 3)
        return {"bytes": size * (live * read + rows * v) + rowwise, "flops": 12 * live * read}
    if kind == "sequence":
        b, n = case["images"], 0.75 * (case["tokens"] - 1)
        k = min(case["removed"], n) / 2
        return {"bytes": b * (8 * (n + 1) + 4 * k + 4 * 9), "flops": b * (8 * n + 30 * k)}
    total, size = 0, 0
    for name, n in _elements(case):
        total, size = total + n, size + n * TYPES[name].itemsize
    if kind == "norm":
        return {"bytes": size + 8, "flops": 2 * total}
    if kind == "clip":
        return {"bytes": 2 * size + 8, "flops": 3 * total}
    p = TYPES[case["param"]].itemsize
    return {"bytes": size + total * (2 * p + 16 + 2 * case["copy"]) + 8, "flops": 16 * total}


# ---------------------------------------------------------------------------
# 64 bits, from the definitions
# ---------------------------------------------------------------------------

def _loss64(lp, old, ref, adv, w, lo, hi, kl, ent_coef, ent):
    """(row losses, d loss / d lp, totals) from numpy arrays of the rows that take part."""
    r = np.exp(lp - old)
    c = np.clip(r, 1 - lo, 1 + hi)
    policy = -np.minimum(r * adv, c * adv)
    flows = r * adv <= c * adv
    k3 = np.expm1(ref - lp) - (ref - lp) if ref is not None else 0 * lp
    row = w * (policy + kl * k3 - ent_coef * ent)
    g = w * (np.where(flows, -r * adv, 0) - (kl * np.expm1(ref - lp) if ref is not None else 0))
    totals = [row.sum(), (w * policy).sum(), (w * k3).sum(), (w * ent).sum(),
              (w * ~flows).sum(), w.sum()]
    return row, g, np.array(totals)


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def _exact_policy(case, s):
    rows, v = case["rows"], case["classes"]
    w, act = _np(s["weights"]), s["actions"].cpu().numpy()
    live = np.flatnonzero((act >= 0) & (w != 0))
    lp, ent = np.zeros(rows), np.zeros(rows)
    grad = torch.zeros(rows, v, dtype=F64, device=DEV)
    step = max(1, (1 << 24) // v)
    legal = s["legal"].cpu().numpy() if s["legal"] is not None else np.full(rows, v)

    def on(values, idx):
        return torch.from_numpy(values[idx].astype(np.int64)).to(DEV)

    for i in range(0, len(live), step):
        idx = live[i:i + step]
        z = s["logits"][torch.from_numpy(idx).to(DEV), :v].double()
        bad = torch.arange(v, device=DEV) >= on(legal, idx)[:, None]
        logq = torch.log_softmax(z.masked_fill(bad, -math.inf), 1)
        h = -torch.special.xlogy(logq.exp(), logq.exp()).sum(1)
        lp[idx] = logq.gather(1, on(act, idx)[:, None])[:, 0].cpu().numpy()
        ent[idx] = h.cpu().numpy()

    def pick(t):
        return None if t is None else _np(t)[live]

    row, g, totals = _loss64(lp[live], pick(s["old"]), pick(s["ref"]), pick(s["adv"]), w[live],
                             s["lo"], s["hi"], case["kl"], case["entropy"], ent[live])
    for i in range(0, len(live), step):
        idx = live[i:i + step]
        at = torch.from_numpy(idx).to(DEV)
        z = s["logits"][at, :v].double()
        bad = torch.arange(v, device=DEV) >= on(legal, idx)[:, None]
        logq = torch.log_softmax(z.masked_fill(bad, -math.inf), 1)
        p = logq.exp()
        gi = torch.from_numpy(g[i:i + step]).to(DEV)[:, None]
        wi = torch.from_numpy(w[idx] * case["entropy"]).to(DEV)[:, None]
        hi = torch.from_numpy(ent[idx]).to(DEV)[:, None]
        d = wi * (torch.special.xlogy(p, p) + p * hi) - gi * p
        d.scatter_add_(1, on(act, idx)[:, None], gi)
        grad[at] = d
    row_all = np.zeros(rows)
    row_all[live] = row
    return {"logp": lp, "entropy": ent, "row_loss": row_all, "totals": totals, "grad": grad}


def _exact_sequence(case, s):
    b = case["images"]
    cu, k, order = (s[x].cpu().numpy() for x in ("cu", "k", "order"))
    scores, w = _np(s["scores"]), _np(s["weights"])
    old, adv, ref = _np(s["old"]), _np(s["adv"]), _np(s["ref"])
    lp, grad = np.zeros(b), np.zeros(len(scores))
    dl = {}
    for i in range(b):
        if k[i] == 0:
            continue
        z = scores[cu[i] + 1:cu[i + 1]]
        seq = order[i, :k[i]]
        stays = np.ones(len(z), bool)
        stays[seq] = False
        rest = np.logaddexp.reduce(z[stays]) if stays.any() else -np.inf
        back = np.logaddexp.accumulate(np.concatenate([[rest], z[seq][::-1]]))[1:][::-1]
        lp[i] = (z[seq] - back).sum()
        upto = np.logaddexp.accumulate(-back)
        d = -np.exp(z + upto[-1])
        d[seq] = 1 - np.exp(z[seq] + upto)
        dl[i] = d
    live = np.array(sorted(dl), dtype=np.int64)
    row_all, totals = np.zeros(b), np.zeros(6)
    if len(live):
        row, g, totals = _loss64(lp[live], old[live], ref[live] if ref is not None else None,
                                 adv[live], w[live], s["lo"], s["hi"], case["kl"], 0.0,
                                 np.zeros(len(live)))
        row_all[live] = row
        for j, i in enumerate(live):
            grad[cu[i] + 1:cu[i + 1]] = g[j] * dl[i]
    return {"logp": lp, "row_loss": row_all, "totals": totals, "grad": grad}


def exact(case, seed):
    kind = case["kind"]
    g = torch.Generator(device=DEV).manual_seed(seed)
    if kind == "policy":
        return _exact_policy(case, _prepare_policy(case, g))
    if kind == "sequence":
        return _exact_sequence(case, _prepare_sequence(case, g))
    s = _prepare_list(case, g)
    squares = sum(float(torch.linalg.vector_norm(x.double()).square()) for x in s["grads"])
    norm = math.sqrt(squares)
    f = min(1.0, s["max_norm"] / norm) if norm else 1.0
    head = torch.tensor([norm, f], dtype=F64)
    if kind == "norm":
        return head
    if kind == "clip":
        return {"norm": head, "clipped": [x.double() * f for x in s["grads"]]}
    t = s["step"] + 1
    d = s["grads"][0].double() * f
    m = torch.lerp(d, s["m"].double(), BETA1)
    v = torch.lerp(d.square(), s["v"].double(), BETA2)
    unit = (m / -math.expm1(t * math.log(BETA1))) / (
        torch.sqrt(v / -math.expm1(t * math.log(BETA2))) + ADAM_EPS)
    p = s["param"].double()
    p = p - s["lr"] * (case["decay"] * p + unit)
    return {"norm": head, "param": p, "m": m, "v": v, "copy": p if case["copy"] else None}
