"""Operators of a policy's rollout and of its matrices' update, as cases that can be timed and
compared.

Four kinds:

* ``logprob``        log-probabilities of given tokens, entropies and the most probable
                     alternatives, from logits;
* ``logprob_grad``   d loss / d logits from d loss / d log-probability and d loss / d entropy;
* ``orthogonalize``  Newton-Schulz iterations that bring a matrix's singular values near 1, over a
                     list of matrices;
* ``muon``           a Muon step over a list of matrices: momentum, orthogonalised update, weights.

``own`` says which form ``run`` computes: false, elementary torch operations in 32 bits; true,
this package's kernels.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
F32, F64, I32 = torch.float32, torch.float64, torch.int32
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
MAX_LOGITS = 4095 * 50001      # of the largest listed loss
STEPS = 5                      # Newton-Schulz iterations
COEF = (3.4445, -4.7750, 2.0315)
MOMENTUM, LR = 0.95, 5e-5      # a backbone or an actor that is tuned further
MAX_FLOPS = 5.3e12             # of the largest listed step, about


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def _logits(name, kind, rows, classes, dtype, pitch, legal, idle, temperature, top, entropy):
    return {"name": name, "kind": kind, "rows": rows, "classes": classes, "dtype": dtype,
            "pitch": pitch, "legal": legal, "idle": idle, "temperature": temperature, "top": top,
            "entropy": entropy}


def _matrices(name, kind, layout, dim, depth, dtype, param="float32", copy=True):
    return {"name": name, "kind": kind, "layout": layout, "dim": dim, "depth": depth, "count": 0,
            "longest": 0, "shape_seed": 0, "dtype": dtype, "param": param, "copy": copy,
            "decay": 0.05, "nesterov": True}


def listed():
    return [
        # the budget head of one rollout batch: 96 counts, feasible ones first, a third of the gates
        # closed; a few microseconds of work
        _logits("logprob_budget_256", "logprob", 256, 96, "float32", 96, True, 0.3, 1.0, 4, True),
        # one new token over a large vocabulary: the row alone does not fill the card
        _logits("logprob_single", "logprob", 1, 131072, "bfloat16", 131072, False, 0.0, 0.7, 20,
                True),
        # a token policy's rollout with padding
        _logits("logprob_tokens_2k", "logprob", 2048, 32000, "bfloat16", 32000, False, 0.15, 1.0, 8,
                True),
        # the largest: an odd number of classes, so that rows start at any alignment
        _logits("logprob_odd_4k", "logprob", 4095, 50001, "float16", 50001, False, 0.05, 1.0, 5,
                True),
        # their gradients, for a loss of the user's own
        _logits("logprob_grad_budget_256", "logprob_grad", 256, 96, "float32", 96, True, 0.3, 1.0,
                0, True),
        _logits("logprob_grad_tokens_2k", "logprob_grad", 2048, 32000, "bfloat16", 32000, False,
                0.15, 1.0, 0, True),
        _logits("logprob_grad_odd_4k", "logprob_grad", 4095, 50001, "float16", 50001, False, 0.05,
                0.7, 0, False),
        # the actor's matrices: twelve of at most 128 rows or columns, latency
        _matrices("orthogonalize_actor", "orthogonalize", "actor", 768, 12, "float32"),
        # the MLPs of two blocks of a large backbone, one tall and one wide matrix each
        _matrices("orthogonalize_mlp", "orthogonalize", "mlp", 1024, 2, "bfloat16"),
        # the actor's step: fp32 masters, bf16 copies for the next rollout
        _matrices("muon_actor", "muon", "actor", 768, 12, "float32"),
        # every matrix of a small backbone's blocks, bf16 gradients
        _matrices("muon_small", "muon", "vit", 384, 12, "bfloat16"),
        # and of a large one's
        _matrices("muon_large", "muon", "vit", 1024, 24, "bfloat16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["logprob", "logprob", "logprob_grad", "orthogonalize", "muon", "muon"])
    if kind.startswith("logprob"):
        dtype = rng.choice(["float32", "bfloat16", "float16"])
        classes = _log_int(rng, 2, 131072)
        most = MAX_LOGITS // classes // (2 if dtype == "float32" else 1)
        rows = _log_int(rng, 1, max(1, min(65536, most)))
        case = {"kind": kind, "rows": rows, "classes": classes, "dtype": dtype,
                "pitch": classes + rng.choice([0, 0, 1, 7, -classes % 64]),
                "legal": rng.random() < 0.3, "idle": rng.choice([0.0, 0.1, 0.4]),
                "temperature": rng.choice([1.0, 0.7, 1.3]),
                "top": rng.choice([0, 1, rng.randint(2, 8), rng.randint(9, 32)]),
                "entropy": rng.random() < 0.7}
        if kind == "logprob_grad":
            case["top"] = 0
        return case
    case = {"kind": kind, "layout": rng.choice(["actor", "vit", "mlp", "ragged", "ragged"]),
            "dim": rng.choice([192, 384, 1024]), "depth": rng.randint(1, 8),
            "count": _log_int(rng, 1, 20), "longest": _log_int(rng, 8, 4096),
            "shape_seed": rng.randrange(1 << 20),
            "dtype": rng.choice(["float32", "bfloat16", "float16"]),
            "param": rng.choice(["float32", "float32", "bfloat16"]), "copy": False,
            "decay": rng.choice([0.0, 0.05]), "nesterov": rng.random() < 0.7}
    case["copy"] = case["param"] == "float32" and rng.random() < 0.7
    if kind == "muon" and rng.random() < 0.2:     # the largest: most blocks of a large backbone
        case.update(layout="vit", dim=1024, depth=rng.randint(9, 22))
    return case


def _shapes(case):
    """(rows, columns) of every matrix of the list."""
    d, depth = case["dim"], case["depth"]
    if case["layout"] == "actor":  # the deployment actor of a backbone of width d, 196 patches
        return [(64, d + 19), (128, d), (128, 128), (128, 128), (128, 128), (128, 128), (256, 128),
                (128, 256), (128, 128), (96, 128), (64, 128), (depth, 128)]
    if case["layout"] == "vit":    # queries, keys, values, projection, MLP
        return ([(d, d)] * 4 + [(4 * d, d), (d, 4 * d)]) * depth
    if case["layout"] == "mlp":
        return [(4 * d, d), (d, 4 * d)] * depth
    rng = random.Random(case["shape_seed"])
    out, flops = [], 0
    while len(out) < case["count"]:
        r, c = _log_int(rng, 1, case["longest"]), _log_int(rng, 1, case["longest"])
        out += [(r, c)]
        flops += _iteration_flops(r, c) * STEPS
        if flops > MAX_FLOPS / 4:
            break
    return out


def _groups(case):
    """[(count, rows, columns)]: the matrices of one shape lie one behind the other."""
    shapes = _shapes(case)
    return [(shapes.count(s), *s) for s in dict.fromkeys(shapes)]


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _prepare_logits(case, g):
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
    tokens = torch.empty(rows, dtype=I32, device=DEV)
    top, logs, ent = (torch.empty(rows, dtype=F64, device=DEV) for _ in range(3))
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
        tokens[r:r + step] = (m / case["temperature"] - (-u.log()).log()).argmax(1).to(I32)
        if case["kind"] == "logprob_grad":      # what the forward has left
            big = m.amax(1, keepdim=True)
            d = (m - big).double() / case["temperature"]
            s = d.exp().sum(1)
            top[r:r + step], logs[r:r + step] = big[:, 0].double(), s.log()
            ent[r:r + step] = s.log() - torch.where(d > -700, d.exp() * d, 0.0).sum(1) / s
    tokens[idle] = -1
    s = {"logits": logits, "legal": legal, "tokens": tokens}
    if case["kind"] == "logprob_grad":
        # gradients of 16 bits with 5 for the exponent are trained with a scaled loss
        scale = (4096.0 if dtype == torch.float16 else 1.0) / max(1, live)
        s["norm"] = torch.where(idle[:, None], 0.0, torch.stack([top, logs], 1)).float()
        s["entropy"] = torch.where(idle, 0.0, ent).float()
        s["dlogp"] = torch.randn(rows, generator=g, device=DEV) * scale
        s["dentropy"] = None
        if case["entropy"]:
            s["dentropy"] = torch.full((rows,), -0.05 * scale, device=DEV)
    return s


def _prepare_matrices(case, g):
    groups = _groups(case)

    def gradient(n, r, c, scale):       # a few strong directions over noise
        k = max(1, min(r, c) // 8)
        left = torch.randn(n, r, k, generator=g, device=DEV)
        right = torch.randn(n, k, c, generator=g, device=DEV)
        noise = torch.randn(n, r, c, generator=g, device=DEV)
        return (left @ right / math.sqrt(k) + 0.3 * noise) * scale

    s = {"groups": groups,
         "grads": [gradient(n, r, c, 1e-3).to(TYPES[case["dtype"]]) for n, r, c in groups]}
    if case["kind"] == "muon":
        s["momentum"] = [gradient(n, r, c, 3e-4) for n, r, c in groups]
        s["param"] = [(torch.randn(n, r, c, generator=g, device=DEV) * 0.02).to(
            TYPES[case["param"]]) for n, r, c in groups]
        s["copy"] = [p.to(torch.bfloat16) for p in s["param"]] if case["copy"] else None
        # the update's size is that of Adam's: 0.2 for every element
        s["scale"] = [0.2 * math.sqrt(max(r, c)) for _, r, c in groups]
        s["clip"] = torch.tensor([0.625, 0.8], device=DEV)      # norm and factor
    return s


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    kind, rows = case["kind"], case.get("rows")
    if kind.startswith("logprob"):
        s = _prepare_logits(case, g)
        if kind == "logprob":
            s["logp"], s["entropy"] = (torch.zeros(rows, device=DEV) for _ in range(2))
            s["norm"] = torch.zeros(rows, 2, device=DEV)
            s["top_logp"] = torch.zeros(rows, case["top"], device=DEV)
            s["top_tokens"] = torch.zeros(rows, case["top"], dtype=I32, device=DEV)
        else:
            s["grad"] = torch.zeros_like(s["logits"])
    else:
        s = _prepare_matrices(case, g)
        if kind == "orthogonalize":
            s["out"] = [torch.zeros_like(x, dtype=torch.bfloat16) for x in s["grads"]]
    s["case"] = case
    if own and "groups" in s:     # the handle that a training program makes once
        import paper_2609_34325_gb300 as P
        if kind == "orthogonalize":
            s["list"] = P.MatrixList(_each(s["grads"]), outs=_each(s["out"]))
        else:
            s["list"] = P.MatrixList(
                _each(s["grads"]), params=_each(s["param"]), momentum=_each(s["momentum"]),
                copies=_each(s["copy"]) if s["copy"] is not None else None,
                scales=[x for x, (n, _, _) in zip(s["scale"], s["groups"]) for _ in range(n)])
    return s


def _each(stacks):
    return [x for t in stacks for x in t.unbind(0)]


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    kind = s["case"]["kind"]
    return {"logprob": _run_logprob, "logprob_grad": _run_logprob_grad,
            "orthogonalize": _run_orthogonalize, "muon": _run_muon}[kind](s)


def _legal_logits(s):
    """fp32 logits with -inf past the legal ones, rows without a token zero; which rows have one;
    which logits count."""
    case, v = s["case"], s["case"]["classes"]
    takes = s["tokens"] >= 0
    use = takes[:, None].expand(-1, v)
    if s["legal"] is not None:
        use = use & (torch.arange(v, device=DEV) < s["legal"][:, None])
    z = torch.where(use, s["logits"][:, :v].float(), -math.inf)
    z[:, 0] = torch.where(takes, z[:, 0], 0.0)
    return z, takes, use


def _run_logprob(s):
    case = s["case"]
    v, k = case["classes"], case["top"]
    if own:
        import paper_2609_34325_gb300 as P
        P.dora_token_logprob(s["logits"], s["tokens"], s["logp"], classes=v, legal=s["legal"],
                             temperature=case["temperature"],
                             entropy=s["entropy"] if case["entropy"] else None, norm=s["norm"],
                             top_logp=s["top_logp"] if k else None,
                             top_tokens=s["top_tokens"] if k else None)
        return {"logp": s["logp"], "entropy": s["entropy"] if case["entropy"] else None,
                "norm": s["norm"], "top_logp": s["top_logp"] if k else None,
                "top_tokens": s["top_tokens"] if k else None}
    z, takes, use = _legal_logits(s)
    m = z.amax(1, keepdim=True)
    d = (z - m) / case["temperature"]
    e = d.exp()
    total = e.sum(1, keepdim=True)
    logs = total.log()
    a = s["tokens"].clamp(min=0).long()[:, None]
    out = {"logp": torch.where(takes, (d.gather(1, a) - logs)[:, 0], 0.0), "entropy": None,
           "norm": torch.where(takes[:, None], torch.cat([m, logs], 1), 0.0), "top_logp": None,
           "top_tokens": None}
    if case["entropy"]:
        mean = torch.where(e > 0, e * d, 0.0).sum(1, keepdim=True) / total
        out["entropy"] = torch.where(takes, (logs - mean)[:, 0], 0.0)
    if k:
        # the largest first, among equal ones the lowest index: keys that are all different
        bits = (z + 0.0).view(I32)
        order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long()
        key = (order << 32) + (0xFFFFFFFF - torch.arange(v, device=DEV))
        best = key.topk(min(k, v), 1).values
        at = 0xFFFFFFFF - (best & 0xFFFFFFFF)
        there = use.gather(1, at)
        pad = (0, k - best.shape[1])
        values = torch.where(there, d.gather(1, at) - logs, -math.inf)
        out["top_logp"] = torch.nn.functional.pad(values, pad, value=-math.inf)
        out["top_tokens"] = torch.nn.functional.pad(torch.where(there, at, -1).to(I32), pad,
                                                    value=-1)
    return out


def _run_logprob_grad(s):
    case = s["case"]
    if own:
        import paper_2609_34325_gb300 as P
        P.dora_token_logprob_grad(s["logits"], s["tokens"], s["norm"], s["grad"],
                                  dlogp=s["dlogp"], dentropy=s["dentropy"], entropy=s["entropy"],
                                  classes=case["classes"], legal=s["legal"],
                                  temperature=case["temperature"])
        return s["grad"][:, :case["classes"]]
    z, takes, use = _legal_logits(s)
    logq = (z - s["norm"][:, :1]) / case["temperature"] - s["norm"][:, 1:]
    p = logq.exp()
    grad = -s["dlogp"][:, None] * p
    if s["dentropy"] is not None:
        more = torch.where(p > 0, p * (logq + s["entropy"][:, None]), 0.0)
        grad = grad - s["dentropy"][:, None] * more
    grad.scatter_add_(1, s["tokens"].clamp(min=0).long()[:, None], s["dlogp"][:, None])
    grad = torch.where(use, grad / case["temperature"], 0.0)
    return grad.to(s["logits"].dtype)


def _newton_schulz(u):
    """A stack of matrices, normalised and iterated on their shorter side."""
    tall = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2) if tall else u
    x = x / x.square().sum((1, 2), keepdim=True).sqrt()
    a, b, c = COEF
    for _ in range(STEPS):
        gram = x @ x.transpose(1, 2)
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.transpose(1, 2) if tall else x


def _run_orthogonalize(s):
    if own:
        import paper_2609_34325_gb300 as P
        P.dora_orthogonalize(s["list"], steps=STEPS)
        return s["out"]
    return [_newton_schulz(x.float()).to(torch.bfloat16) for x in s["grads"]]


def _run_muon(s):
    case = s["case"]
    if own:
        import paper_2609_34325_gb300 as P
        P.dora_muon_step(s["list"], LR, momentum=MOMENTUM, nesterov=case["nesterov"],
                         weight_decay=case["decay"], steps=STEPS, clip=s["clip"])
        return {k: s[k] for k in ("param", "momentum", "copy")}

    def step(grad, m, p, scale):
        d = grad.float() * s["clip"][1]
        m = MOMENTUM * m + (1 - MOMENTUM) * d
        u = (1 - MOMENTUM) * d + MOMENTUM * m if case["nesterov"] else m
        p = p.float() * (1 - LR * case["decay"]) - (LR * scale) * _newton_schulz(u)
        return m, p

    both = [step(*x) for x in zip(s["grads"], s["momentum"], s["param"], s["scale"])]
    s["momentum"] = [m for m, _ in both]
    s["param"] = [p.to(TYPES[case["param"]]) for _, p in both]
    s["copy"] = [p.to(torch.bfloat16) for _, p in both] if case["copy"] else None
    return {k: s[k] for k in ("param", "momentum", "copy")}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def _iteration_flops(r, c):
    """One Newton-Schulz iteration, the two symmetric products by half."""
    m, n = min(r, c), max(r, c)
    return m * m * n + m ** 3 + 2 * m * m * n


def work(case):
    kind = case["kind"]
    if kind.startswith("logprob"):
        rows, v, size = case["rows"], case["classes"], TYPES[case["dtype"]].itemsize
        live = rows - int(case["idle"] * rows)
        read = v / 2 if case["legal"] else v           # legal counts are spread over 1..v
        rowwise = 4 * rows * (4 + bool(case["legal"]) + bool(case["entropy"]) + 2 * case["top"])
        if kind == "logprob_grad":
            rowwise += size * rows * v
        return {"bytes": size * live * read + rowwise, "flops": 8 * live * read}
    n = sum(r * c for r, c in _shapes(case))
    size = TYPES[case["dtype"]].itemsize + 2
    if kind == "muon":
        size += 8 + 2 * TYPES[case["param"]].itemsize - 2 + 2 * case["copy"]
    return {"bytes": n * size, "flops": STEPS * sum(_iteration_flops(r, c)
                                                    for r, c in _shapes(case))}


# ---------------------------------------------------------------------------
# 64 bits, from the definitions
# ---------------------------------------------------------------------------

def _chunks(case, s):
    """(rows, scaled logits in 64 bits with -inf past the legal ones) of the rows that count."""
    live = torch.nonzero(s["tokens"] >= 0)[:, 0]
    v = case["classes"]
    for at in live.split(max(1, (1 << 24) // v)):
        z = s["logits"][at, :v].double() / case["temperature"]
        if s["legal"] is not None:
            z[torch.arange(v, device=DEV) >= s["legal"][at, None]] = -math.inf
        yield at, z


def _exact_logprob(case, s):
    rows, k = case["rows"], case["top"]
    logp, ent = (torch.zeros(rows, dtype=F64, device=DEV) for _ in range(2))
    norm = torch.zeros(rows, 2, dtype=F64, device=DEV)
    best = torch.full((rows, k), -math.inf, dtype=F64, device=DEV)
    ids = torch.full((rows, k), -1, dtype=I32, device=DEV)
    for at, z in _chunks(case, s):
        q = torch.log_softmax(z, 1)
        logp[at] = q.gather(1, s["tokens"][at].long()[:, None])[:, 0]
        ent[at] = -torch.special.xlogy(q.exp(), q.exp()).sum(1)
        norm[at, 0] = z.amax(1) * case["temperature"]
        norm[at, 1] = torch.logsumexp(z, 1) - z.amax(1)
        if k:
            order = (z + 0.0).sort(dim=1, descending=True, stable=True).indices[:, :k]
            w = q.gather(1, order)
            best[at, :w.shape[1]] = w
            ids[at, :w.shape[1]] = torch.where(w > -math.inf, order, -1).to(I32)
    return {"logp": logp, "entropy": ent if case["entropy"] else None, "norm": norm,
            "top_logp": best if k else None, "top_tokens": ids if k else None}


def _exact_logprob_grad(case, s):
    grad = torch.zeros(case["rows"], case["classes"], dtype=F64, device=DEV)
    for at, z in _chunks(case, s):
        one = torch.zeros_like(z).scatter_(1, s["tokens"][at].long()[:, None], 1.0)
        m, logs = s["norm"][at].double().unbind(1)
        p = torch.exp(z - (m / case["temperature"] + logs)[:, None])
        d = s["dlogp"][at].double()[:, None] * (one - p)
        if s["dentropy"] is not None:
            h = s["entropy"][at].double()[:, None]
            d -= s["dentropy"][at].double()[:, None] * (torch.special.xlogy(p, p) + p * h)
        grad[at] = d / case["temperature"]
    return grad


def _exact_orthogonal(u):
    """The iteration's polynomial of odd powers, applied to a matrix from its right side."""
    u = u.double()
    if u.shape[0] < u.shape[1]:
        return _exact_orthogonal(u.t()).t()
    x = u / torch.linalg.vector_norm(u)
    eye = torch.eye(u.shape[1], dtype=F64, device=DEV)
    for _ in range(STEPS):
        g = x.t() @ x
        x = x @ (COEF[0] * eye + g @ (COEF[1] * eye + COEF[2] * g))
    return x


def exact(case, seed):
    kind = case["kind"]
    g = torch.Generator(device=DEV).manual_seed(seed)
    if kind.startswith("logprob"):
        s = _prepare_logits(case, g)
        return _exact_logprob(case, s) if kind == "logprob" else _exact_logprob_grad(case, s)
    s = _prepare_matrices(case, g)
    if kind == "orthogonalize":
        return [torch.stack([_exact_orthogonal(x) for x in t]) for t in s["grads"]]
    out = {"param": [], "momentum": [], "copy": [] if case["copy"] else None}
    for t, m, p, scale in zip(s["grads"], s["momentum"], s["param"], s["scale"]):
        d = t.double() * float(s["clip"][1])
        m = torch.lerp(d, m.double(), MOMENTUM)
        u = torch.lerp(d, m, MOMENTUM) if case["nesterov"] else m
        o = torch.stack([_exact_orthogonal(x) for x in u])
        p = p.double() - LR * (case["decay"] * p.double() + scale * o)
        for name, value in (("param", p), ("momentum", m), ("copy", p)):
            if out[name] is not None:
                out[name].append(value)
    return out
