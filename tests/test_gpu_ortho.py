"""GPU parity of the orthogonalised updates and the Muon step against the fp64 oracle.

Bounds.  An iteration rounds four matrices to fp16 (X twice, F, G), each 2^-12 / sqrt(3) =
1.4e-4 of itself in the 2-norm; their gains, |d p(s) / d| of the quintic for singular
values up to 1.21, are at most 3.1.  Five iterations in quadrature: sqrt(20) 3.1 1.4e-4 =
1.9e-3, and as much again for what later iterations make of it: 4e-3 in the 2-norm.  The
output's own rounding is 2^-8 at most for each value (bf16).  More iterations than five add
their share: sqrt(steps / 5).  Few values may miss the average: 1 + 4 / sqrt(count)."""
import numpy as np
import pytest
import torch

import __graft_entry__ as G
import oracle as O
import paper_2609_34325_gb300 as P
from helpers import dev

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
ROUND = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}
SHAPES = [(1, 1), (1, 9), (9, 1), (3, 50), (64, 64), (100, 37), (128, 128), (129, 128), (128, 129),
          (64, 787), (128, 768), (256, 128), (300, 200), (257, 511), (384, 384), (640, 256),
          (130, 1100), (1000, 390)]


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    G.build()
    P.load_library()
    torch.cuda.set_device(0)


def _np(t):
    return t.detach().double().cpu().numpy()


def _random(shapes, dtype, seed, scale=1.0, strong=False, shift=0):
    """Gaussian matrices; strong: a few directions over noise."""
    g = torch.Generator(device=dev()).manual_seed(seed)
    out = []
    for r, c in shapes:
        x = torch.randn(r, c, generator=g, device=dev())
        if strong:
            k = max(1, min(r, c) // 8)
            x = 0.2 * x + torch.randn(r, k, generator=g, device=dev()) @ torch.randn(
                k, c, generator=g, device=dev()) / k ** 0.5
        flat = torch.empty(r * c + shift, dtype=dtype, device=dev())
        y = flat[shift:].view(r, c)
        y.copy_((x * scale).to(dtype))
        out.append(y)
    return out


def _bound(count, steps=5):
    return 4e-3 * max(1.0, (steps / 5) ** 0.5) * (1 + 4 / count ** 0.5)


def _off(got, ref):
    return np.linalg.norm(got - ref) / max(np.linalg.norm(ref), 1e-300)


def _orthogonalize(grads, steps=5, shift=0, **more):
    outs = []
    for x in grads:
        flat = torch.full((x.numel() + shift,), 7.0, dtype=BF16, device=dev())
        outs.append(flat[shift:].view(x.shape))
    lst = P.MatrixList(grads, outs=outs)
    P.dora_orthogonalize(lst, steps=steps, **more)
    torch.cuda.synchronize()
    return outs, lst


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("strong,shift", [(False, 0), (True, 1)])
def test_orthogonalize_a_list(dtype, strong, shift):
    grads = _random(SHAPES, dtype, 1, 1e-2, strong, shift)
    status = torch.zeros(1, dtype=torch.int32, device=dev())
    outs, _ = _orthogonalize(grads, shift=shift, status=status)
    assert int(status) == 0
    for x, o in zip(grads, outs):
        ref = O.newton_schulz(_np(x))
        assert _off(_np(o), ref) <= _bound(ref.size) + 2.0 ** -8, x.shape


@pytest.mark.parametrize("shape", SHAPES)
def test_orthogonalize_one_matrix(shape):
    (x,), steps = _random([shape], F32, 2), 1 + sum(shape) % 6
    (o,), _ = _orthogonalize([x], steps)
    ref = O.newton_schulz(_np(x), steps)
    assert _off(_np(o), ref) <= _bound(ref.size, steps) + 2.0 ** -8


def test_orthogonalize_larger_matrices():
    for shape in ((1024, 1024), (2048, 700), (520, 4100)):
        (x,) = _random([shape], BF16, 3, 1.0, True)
        (o,), _ = _orthogonalize([x])
        assert _off(_np(o), O.newton_schulz(_np(x))) <= _bound(x.numel()) + 2.0 ** -8


@pytest.mark.parametrize("scale", [1e-42, 1e-38, 1e-30, 1e-10, 1e10, 1e30, 1e37])
def test_scale_of_the_update_does_not_matter(scale):
    grads = _random([(70, 200), (200, 70), (1, 5)], F32, 4, scale)
    outs, _ = _orthogonalize(grads)
    for x, o in zip(grads, outs):
        # of the subnormal values that there are
        ref = O.newton_schulz(_np(x))
        assert _off(_np(o), ref) <= _bound(ref.size) + 2.0 ** -8


def test_values_of_very_different_sizes():
    (x,) = _random([(150, 260)], F32, 5)
    x[:75] *= 1e-20
    x[3] *= 1e15
    (o,), _ = _orthogonalize([x])
    ref = O.newton_schulz(_np(x))
    assert _off(_np(o), ref) <= _bound(ref.size) + 2.0 ** -8


def test_zeros_and_what_is_not_finite():
    grads = _random([(40, 300), (300, 40), (64, 64), (9, 9), (200, 130)], F32, 6)
    grads[0].zero_()
    grads[1][7, 3] = float("inf")
    grads[3][8, 8] = float("nan")
    outs, _ = _orthogonalize(grads)
    assert not outs[0].any()
    assert bool(torch.isnan(outs[1]).all()) and bool(torch.isnan(outs[3]).all())
    for i in (2, 4):
        assert _off(_np(outs[i]), O.newton_schulz(_np(grads[i]))) <= _bound(4096) + 2.0 ** -8


# Up to 32 rows or columns X, F and G have 22 bits: an iteration's four roundings of 2^-22 (the
# sums' among them) grow by 3.4445 at most in each of those that follow: 4 2^-22 (1 + 3.4 + .. +
# 3.4445^4) = 1.9e-4.  Weights of 0, a rate of 1 and no momentum show the result in 32 bits.
@pytest.mark.parametrize("shape", [(1, 1), (1, 2), (2, 1), (1, 40), (2, 2), (2, 5), (3, 3), (50, 3),
                                   (5, 5), (8, 9), (16, 16), (32, 32), (32, 33), (20, 700),
                                   (700, 12), (32, 2048), (1500, 17)])
def test_few_rows_are_exact(shape):
    grads = _random([shape] * 20, F32, 81)
    params = [torch.zeros_like(x) for x in grads]
    lst = P.MatrixList(grads, params=params, momentum=[torch.zeros_like(x) for x in grads],
                       scales=[1.0] * 20)
    P.dora_muon_step(lst, 1.0, momentum=0.0)
    torch.cuda.synchronize()
    for x, p in zip(grads, params):
        assert _off(-_np(p), O.newton_schulz(_np(x))) <= 2e-4


def test_low_rank_updates():
    g = torch.Generator(device=dev()).manual_seed(7)
    for r, c, k in ((200, 300, 1), (300, 200, 5), (128, 640, 2)):
        x = torch.randn(r, k, generator=g, device=dev()) @ torch.randn(k, c, generator=g,
                                                                     device=dev())
        (o,), _ = _orthogonalize([x])
        # fp32's rounding of x is a noise of 2^-24 that the iteration raises by 3.4445^5 = 485
        ref = O.newton_schulz(_np(x))
        assert _off(_np(o), ref) <= _bound(ref.size) + 2.0 ** -8


def _muon(shapes, gt, pt, seed, shift=0):
    g = _random(shapes, gt, seed, 1e-3, True, shift)
    m = _random(shapes, F32, seed + 1, 1e-3, True, shift)
    p = _random(shapes, pt, seed + 2, 0.02, False, shift)
    return g, m, p


def _check_step(g, m0, p0, m, p, copies, kw, scales, factor):
    for i in range(len(g)):
        pr, mr = O.muon_step(p0[i], m0[i], _np(g[i]), kw["lr"], kw["momentum"], kw["nesterov"],
                             kw["weight_decay"], scales[i], kw.get("steps", 5), factor)
        gi = np.abs(factor * _np(g[i]))
        assert np.all(np.abs(_np(m[i]) - mr) <= 2.0 ** -21 * (np.abs(m0[i]) + gi) + 1e-40)
        o = (p0[i] * (1 - kw["lr"] * kw["weight_decay"]) - pr)      # lr scale NS(u)
        diff = _np(p[i]) - pr
        r = ROUND[p[i].dtype] + 2.0 ** -22
        rounding = r * np.linalg.norm(pr) + 1e-9
        assert np.linalg.norm(diff) <= _bound(pr.size) * np.linalg.norm(o) + rounding
        if copies is not None:
            want = p[i].to(BF16) if p[i].dtype == F32 else None
            if want is not None:
                assert torch.equal(copies[i], want)
            assert np.linalg.norm(_np(copies[i]) - pr) <= _bound(pr.size) * np.linalg.norm(o) + (
                2.0 ** -8 + r) * np.linalg.norm(pr) + 1e-9


@pytest.mark.parametrize("gt", [F32, BF16, F16])
@pytest.mark.parametrize("pt", [F32, BF16, F16])
@pytest.mark.parametrize("nesterov,shift", [(True, 0), (False, 1)])
def test_muon_steps(gt, pt, nesterov, shift):
    g, m, p = _muon(SHAPES, gt, pt, 11, shift)
    copies = [torch.zeros(t.numel() + shift, dtype=BF16, device=dev())[shift:].view(t.shape)
              for t in p]
    scales = [0.5 + 0.1 * i for i in range(len(g))]
    lst = P.MatrixList(g, params=p, momentum=m, copies=copies, scales=scales)
    clip = torch.tensor([2.0, 0.25], device=dev())
    for step in range(2):
        m0, p0 = [_np(t) for t in m], [_np(t) for t in p]
        kw = dict(lr=2e-2, momentum=0.9, nesterov=nesterov, weight_decay=0.1)
        P.dora_muon_step(lst, clip=clip if step else None, **kw)
        torch.cuda.synchronize()
        _check_step(g, m0, p0, m, p, copies, kw, scales, 0.25 if step else 1.0)


def test_muon_default_scales_and_no_momentum():
    g, m, p = _muon([(30, 90), (90, 30)], F32, F32, 21)
    lst = P.MatrixList(g, params=p, momentum=m)
    assert lst.scales == [1.0, 3.0 ** 0.5]
    m0, p0 = [_np(t) for t in m], [_np(t) for t in p]
    kw = dict(lr=1e-2, momentum=0.0, nesterov=True, weight_decay=0.0)
    P.dora_muon_step(lst, **kw)
    torch.cuda.synchronize()
    _check_step(g, m0, p0, m, p, None, kw, lst.scales, 1.0)


def test_muon_skips_a_norm_that_is_not_finite():
    g, m, p = _muon([(150, 40), (20, 20)], F32, F32, 31)
    copies = [t.to(BF16) for t in p]
    lst = P.MatrixList(g, params=p, momentum=m, copies=copies)
    vectors = torch.randn(50, device=dev())
    everything = P.ParamList([*g, vectors])
    norm = torch.zeros(2, device=dev())
    before = [t.clone() for t in m + p + copies]
    for value in (np.inf, np.nan):
        vectors[3] = value                       # in another tensor of the same step
        P.dora_grad_norm(everything, 1.0, norm)
        P.dora_muon_step(lst, 1e-2, clip=norm)
        torch.cuda.synchronize()
        for t, b in zip(m + p + copies, before):
            assert torch.equal(t, b)
    vectors[3] = 0.0
    P.dora_grad_norm(everything, 1e-3, norm)
    m0, p0 = [_np(t) for t in m], [_np(t) for t in p]
    P.dora_muon_step(lst, 1e-2, clip=norm)
    torch.cuda.synchronize()
    kw = dict(lr=1e-2, momentum=0.95, nesterov=True, weight_decay=0.0)
    _check_step(g, m0, p0, m, p, copies, kw, lst.scales, float(norm[1]))


def test_same_bits_streams_and_graphs():
    shapes = [(128, 128), (64, 787), (390, 260), (500, 700)]
    runs = []
    for how in range(3):
        g, m, p = _muon(shapes, BF16, F32, 41)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        if how == 0:
            lst = P.MatrixList(g, params=p, momentum=m)
            for _ in range(3):
                P.dora_muon_step(lst, 1e-2)
        else:
            lst = P.MatrixList(g, params=p, momentum=m, stream=side)
            if how == 1:
                for _ in range(3):
                    P.dora_muon_step(lst, 1e-2, stream=side)
            else:
                graph = torch.cuda.CUDAGraph()
                torch.cuda.synchronize()
                with torch.cuda.stream(side):
                    with torch.cuda.graph(graph, stream=side):
                        P.dora_muon_step(lst, 1e-2)
                for _ in range(3):
                    graph.replay()
        torch.cuda.synchronize()
        runs.append(m + p)
    for a, b, c in zip(*runs):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_the_same_bits_every_time():
    # odd numbers of blocks, whose last pair has one row block only; who takes which tile, and
    # what is waited for, differs from call to call
    grads = _random([(257, 511), (300, 200), (390, 260), (640, 700), (130, 1100), (900, 129)] * 2,
                    BF16, 55)
    outs, lst = _orthogonalize(grads)
    first = [o.clone() for o in outs]
    for _ in range(40):
        for o in outs:
            o.zero_()
        P.dora_orthogonalize(lst)
        torch.cuda.synchronize()
        assert all(torch.equal(o, f) for o, f in zip(outs, first))
    for x, o in zip(grads, outs):
        assert _off(_np(o), O.newton_schulz(_np(x))) <= _bound(x.numel()) + 2.0 ** -8


def test_a_matrix_does_not_depend_on_its_list():
    grads = _random([(300, 200), (64, 787), (200, 300), (128, 128)], BF16, 51)
    together, _ = _orthogonalize(grads)
    for x, o in zip(grads, together):
        (alone,), _ = _orthogonalize([x])
        assert torch.equal(alone, o)


@pytest.mark.parametrize("small,large", [(6, 2), (200, 1), (40, 30)])
def test_small_matrices_beside_large_ones(small, large):
    # both kinds in a list run at the same time; steps one behind the other, and what reads the
    # weights after them, wait for both
    shapes = [(100, 37), (64, 787), (9, 1500), (128, 128)] * small + [(640, 700), (257, 511)] * large
    shapes = shapes[:small] + shapes[4 * small:]

    def steps(lists):
        g, m, p = _muon(shapes, BF16, F32, 43)
        seen = []
        made = [P.MatrixList([g[i] for i in k], params=[p[i] for i in k],
                             momentum=[m[i] for i in k]) for k in lists]
        for _ in range(4):
            for lst in made:
                P.dora_muon_step(lst, 1e-2)
            seen.append([x.clone() for x in p])
            for x, y in zip(g, p):                 # gradients of the new weights
                x.copy_(y * 0.1 + x * 0.9)
        torch.cuda.synchronize()
        return [x for r in seen for x in r] + m

    every = range(len(shapes))
    together = steps([every])
    apart = steps([[i for i in every if i < small], [i for i in every if i >= small]])
    assert all(torch.equal(a, b) for a, b in zip(together, apart))


def test_what_lies_beside_the_matrices_stays():
    flat = torch.full((4000,), 7.0, dtype=BF16, device=dev())
    out = flat[101:101 + 33 * 65].view(33, 65)
    (x,) = _random([(33, 65)], F32, 61)
    P.dora_orthogonalize(P.MatrixList([x], outs=[out]))
    torch.cuda.synchronize()
    assert bool((flat[:101] == 7.0).all()) and bool((flat[101 + 33 * 65:] == 7.0).all())
    assert not bool((out == 7.0).any())


def test_another_current_device_is_refused(monkeypatch):
    (x,) = _random([(8, 12)], F32, 72)
    lst = P.MatrixList([x], params=[x.clone()], momentum=[x.clone()], outs=[x.to(BF16)])
    monkeypatch.setattr(P, "_raw_device", lambda: 1)
    for call in (lambda: P.MatrixList([x], outs=[x.to(BF16)]), lambda: P.dora_orthogonalize(lst),
                 lambda: P.dora_muon_step(lst, 0.1)):
        with pytest.raises(ValueError, match="current device"):
            call()


# The longest side; and more than 2^31 elements.  An X X^T of n columns is added up in n / 16
# steps, each cut off to 32 bits, half of 2^-23 of what there is on average: n 2^-28 of itself at
# most, of which the iterations, |b s^2 + 2 c s^4| <= 1.8 each, make less than n 2^-26.
@pytest.mark.parametrize("m,n", [(130, 1 << 18), (8200, 1 << 18)])
def test_long_matrices(m, n):
    # What the iteration makes of X0 is M X0, with M a polynomial of A = X0 X0^T, here from fp32
    # products of few columns added in 64 bits
    x = torch.empty(m, n, dtype=BF16, device=dev())
    for r in range(m):
        x[r].normal_(generator=torch.Generator(device=dev()).manual_seed(r))
    x[:60] += x[60:120]
    before = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    gram = torch.zeros(m, m, dtype=torch.float64, device=dev())
    for c in range(0, n, 4096):
        y = x[:, c:c + 4096].float()
        gram += (y @ y.t()).double()
    size = torch.trace(gram).sqrt()
    gram = (gram / (size * size)).float()
    a, b, c = O.NS_COEF
    eye = torch.eye(m, device=dev())
    poly = eye
    for _ in range(5):
        p = poly @ gram @ poly.t()
        poly = (a * eye + b * p + c * p @ p) @ poly
    out = torch.empty_like(x)
    P.dora_orthogonalize(P.MatrixList([x], outs=[out]))
    torch.cuda.synchronize()
    for c in (0, n // 2, n - 1000):
        want = poly @ x[:, c:c + 1000].float() / size.float()
        off = float((out[:, c:c + 1000].float() - want).norm() / want.norm())
        assert off <= _bound(m * 1000) + n * 2.0 ** -26 + 2.0 ** -8, (c, off)
    torch.backends.cuda.matmul.allow_tf32 = before


def test_refusals():
    (x,) = _random([(8, 12)], F32, 71)
    bf = x.to(BF16)
    for bad in (dict(grads=[x[:, ::2]]), dict(grads=[x.t()]), dict(grads=[x[0]]),
                dict(grads=[x.double()]), dict(grads=[x], outs=[x]), dict(grads=[x], outs=[bf[:4]]),
                dict(grads=[x], outs=[bf.view(12, 8)]), dict(grads=[x], params=[x]),
                dict(grads=[x], params=[x], momentum=[bf]), dict(grads=[x], copies=[bf]),
                dict(grads=[x], outs=[bf], scales=[float("nan")]),
                dict(grads=[x[:0]], outs=[bf[:0]]), dict(grads=[x, x], outs=[bf])):
        with pytest.raises((TypeError, ValueError)):
            P.MatrixList(**bad)
    with pytest.raises(ValueError):          # buffers that overlap
        P.MatrixList([x], params=[x], momentum=[x.clone()])
    with pytest.raises(ValueError):
        P.MatrixList([x, x], outs=[bf, bf])
    only_outs = P.MatrixList([x], outs=[bf.clone()])
    only_params = P.MatrixList([x], params=[x.clone()], momentum=[x.clone()])
    with pytest.raises(P.DoraError):
        P.dora_muon_step(only_outs, 0.1)
    with pytest.raises(P.DoraError):
        P.dora_orthogonalize(only_params)
    for kw in (dict(lr=float("nan")), dict(lr=0.1, momentum=1.0), dict(lr=0.1, weight_decay=-1.0),
               dict(lr=0.1, steps=0), dict(lr=0.1, steps=33)):
        with pytest.raises(P.DoraError):
            P.dora_muon_step(only_params, **kw)
    with pytest.raises(ValueError):
        P.dora_muon_step(only_params, 0.1, clip=torch.zeros(1, device=dev()))
    with pytest.raises(TypeError):
        P.dora_muon_step(only_params, 0.1, clip=torch.zeros(2))
