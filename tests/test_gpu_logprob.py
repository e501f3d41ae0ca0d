"""GPU parity of token log-probabilities, entropies, alternatives and their gradient,
against the fp64 oracle.

Bounds.  A thread adds up to n / 512 exponentials (two sums, a row over 256 threads at
least where it is long), each 2^-22 of itself off, its exponent 2^-22 of |d| / T; a
shuffle tree follows.  So s is off by e_s = (n / 512 + 24) 2^-24 + 2^-22 (1 + E|d| / T),
ln s by that; l adds 2^-22 |d_a| / T, the entropy the same errors of t / (T s).  A gradient's
p_j is off by 2^-22 (1 + |d_j| / T + |ln s|) of itself, and by what (m, ln s, H) are; then it is
rounded to its type."""
import numpy as np
import pytest
import torch

import __graft_entry__ as G
import oracle as O
import paper_2609_34325_gb300 as P
from helpers import dev

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
I32 = torch.int32
ROUND = {BF16: (2.0 ** -8, 1e-38), F16: (2.0 ** -11, 2.0 ** -25), F32: (2.0 ** -24, 1e-38)}


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    G.build()
    P.load_library()
    torch.cuda.set_device(0)


def _np(t):
    return t.detach().double().cpu().numpy()


def _logits(rows, classes, dtype, seed, pad=0, shift=0, step=0.0, scale=2.5):
    """[rows, classes] logits in a buffer of NaN: rows `pad` apart, `shift` elements in;
    `step`: multiples of it, so that many are equal."""
    g = torch.Generator(device=dev()).manual_seed(seed)
    ld = classes + pad
    flat = torch.full((shift + rows * ld + 16,), float("nan"), dtype=dtype, device=dev())
    z = flat[shift:shift + rows * ld].view(rows, ld)[:, :classes]
    v = torch.randn(rows, classes, generator=g, device=dev()) * scale
    z.copy_((torch.round(v / step) * step if step else v).to(dtype))
    return z


def _forward(z, tokens, legal=None, temperature=1.0, top=0, status=None, stream=None):
    rows = z.shape[0]
    o = {"logp": torch.full((rows,), 7.0, device=dev()) if tokens is not None else None,
         "entropy": torch.full((rows,), 7.0, device=dev()),
         "norm": torch.full((rows, 2), 7.0, device=dev()),
         "top_logp": torch.full((rows, top), 7.0, device=dev()),
         "top_tokens": torch.full((rows, top), 7, dtype=I32, device=dev())}
    P.dora_token_logprob(z, tokens, o["logp"], legal=legal, temperature=temperature,
                         entropy=o["entropy"], norm=o["norm"], top_logp=o["top_logp"],
                         top_tokens=o["top_tokens"], status=status, stream=stream)
    return o


def _check(z, tokens, o, legal=None, temperature=1.0):
    zz = _np(z)
    tk = None if tokens is None else tokens.cpu().numpy()
    lg = None if legal is None else legal.cpu().numpy()
    top = o["top_tokens"].shape[1]
    ref = O.token_logprob(zz, tk, lg, temperature, top)
    n = zz.shape[1]
    with np.errstate(invalid="ignore", divide="ignore"):
        d = np.abs(zz - ref["norm"][:, :1]) / temperature
        d = np.where(np.isfinite(d), d, 0.0)
        p = np.exp(-d)
        if lg is not None:
            p[np.arange(n) >= lg[:, None]] = 0
        mean_d = (p * d).sum(1) / np.maximum(p.sum(1), 1e-300)
    e_s = (n / 512 + 24) * 2.0 ** -24 + 2.0 ** -22 * (1 + mean_d)
    ls = np.abs(ref["norm"][:, 1])
    takes = (np.ones(len(zz), bool) if tk is None else tk >= 0) & (
        np.ones(len(zz), bool) if lg is None else lg > 0)
    assert np.array_equal(_np(o["norm"])[:, 0], ref["norm"][:, 0])
    tol = e_s + 2.0 ** -22 * (1 + ls)
    assert np.all(np.abs(_np(o["norm"])[:, 1] - ref["norm"][:, 1]) <= tol)
    assert np.all(np.abs(_np(o["entropy"]) - ref["entropy"]) <= tol + 3 * e_s * (1 + mean_d))
    if tk is not None:
        at = np.where(takes, tk, 0)
        da = d[np.arange(len(zz)), at]
        got = _np(o["logp"])
        same = got == ref["logp"]                              # -inf among them
        with np.errstate(invalid="ignore"):
            assert np.all(same | (np.abs(got - ref["logp"]) <= tol + 2.0 ** -22 * da))
        assert not got[~takes].any()
    assert np.array_equal(o["top_tokens"].cpu().numpy(), ref["top_tokens"])
    got, there = _np(o["top_logp"]), ref["top_tokens"] >= 0
    da = np.take_along_axis(d, np.maximum(ref["top_tokens"], 0), 1)
    with np.errstate(invalid="ignore"):
        off = np.abs(got - ref["top_logp"]) <= tol[:, None] + 2.0 ** -22 * da
    assert np.all(np.where(there, off, np.isneginf(got)))
    return ref


SIZES = [(1, 1), (3, 2), (5, 7), (256, 96), (33, 130), (17, 257), (9, 1000), (40, 1024), (6, 2047),
         (5, 4099), (3, 16384), (2, 50001), (1, 131072), (700, 300)]


@pytest.mark.parametrize("rows,classes", SIZES)
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("pad,shift,top", [(0, 0, 5), (1, 3, 32), (64, 1, 1), (3, 0, 0)])
def test_forward(rows, classes, dtype, pad, shift, top):
    z = _logits(rows, classes, dtype, rows + classes, pad, shift)
    tokens = torch.randint(0, classes, (rows,), device=dev(), dtype=I32)
    o = _forward(z, tokens, top=top, temperature=1.0 if pad else 0.7)
    torch.cuda.synchronize()
    _check(z, tokens, o, temperature=1.0 if pad else 0.7)


@pytest.mark.parametrize("classes", [5, 96, 515, 3000, 20000])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("top", [3, 32])
def test_legal_prefixes_and_rows_without_a_token(classes, dtype, top):
    rows = 37
    z = _logits(rows, classes, dtype, classes, 5, 2)
    g = torch.Generator(device=dev()).manual_seed(1)
    legal = torch.randint(0, classes + 1, (rows,), generator=g, device=dev(), dtype=I32)
    legal[:4] = torch.tensor([0, 1, classes, 2], device=dev())
    tokens = (torch.rand(rows, generator=g, device=dev()) * legal).to(I32)
    tokens[legal == 0] = -1
    tokens[5::7] = -100
    for r in range(rows):
        z[r, int(legal[r]):] = float("nan")        # not read
        if tokens[r] < 0:
            z[r] = float("nan")
    status = torch.zeros(1, dtype=I32, device=dev())
    o = _forward(z, tokens, legal, top=top, status=status)
    torch.cuda.synchronize()
    _check(torch.nan_to_num(z), tokens, o, legal)
    assert int(status) == 0
    # without tokens every row with legal logits takes part
    z = torch.nan_to_num(z)
    o = _forward(z, None, legal, top=top, status=status)
    torch.cuda.synchronize()
    _check(z, None, o, legal)
    assert int(status) == 0


@pytest.mark.parametrize("classes", [40, 1000, 5000, 40000])
@pytest.mark.parametrize("step", [0.5, 4.0, 100.0])
@pytest.mark.parametrize("top", [1, 8, 32])
def test_equal_logits_come_by_index(classes, step, top):
    z = _logits(6, classes, BF16, 3, 1, 0, step)
    z[2] = -0.0
    z[2, ::3] = 0.0
    tokens = torch.zeros(6, dtype=I32, device=dev())
    o = _forward(z, tokens, top=top)
    torch.cuda.synchronize()
    _check(z, tokens, o)


@pytest.mark.parametrize("order", [1, -1])
@pytest.mark.parametrize("classes", [200, 2048, 30011])
def test_sorted_rows(order, classes):
    z = torch.linspace(-9, 9, classes, device=dev())[None].repeat(3, 1)
    z = (z.flip(1) if order < 0 else z).contiguous()
    tokens = torch.full((3,), classes - 1, dtype=I32, device=dev())
    o = _forward(z, tokens, top=32)
    torch.cuda.synchronize()
    _check(z, tokens, o)


@pytest.mark.parametrize("classes", [9, 700, 6000, 40000])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_masked_logits(classes, dtype):
    low = torch.finfo(dtype).min
    z = _logits(5, classes, dtype, 8)
    z[0] = float("-inf")
    z[0, classes // 2] = 1.0                       # one logit left: certain
    z[1, 1:] = low
    z[2, ::2] = float("-inf")
    z[3] = low                                     # all the same: uniform
    z[4, 3:] = float("-inf")
    tokens = torch.tensor([classes // 2, 0, 0, 1, 0], dtype=I32, device=dev())
    o = _forward(z, tokens, top=6)
    torch.cuda.synchronize()
    _check(z, tokens, o)
    assert float(o["logp"][0]) == 0.0 and float(o["entropy"][0]) == 0.0
    assert np.isneginf(float(o["logp"][2]))
    assert o["top_tokens"][0].tolist() == [classes // 2] + [-1] * 5
    assert abs(float(o["entropy"][3]) - np.log(classes)) < 1e-4


@pytest.mark.parametrize("classes", [6, 300, 5000, 40000])
def test_rows_that_are_not_finite(classes):
    z = _logits(6, classes, F32, 9)
    z[1, classes - 1] = float("nan")
    z[2, 0] = float("inf")
    z[3] = float("-inf")
    z[4, :] = float("inf")
    tokens = torch.ones(6, dtype=I32, device=dev())
    status = torch.zeros(1, dtype=I32, device=dev())
    o = _forward(z, tokens, top=4, status=status)
    torch.cuda.synchronize()
    for r in (1, 2, 3, 4):
        assert np.isnan(_np(o["logp"])[r]) and np.isnan(_np(o["entropy"])[r])
        assert np.isnan(_np(o["norm"])[r]).all() and np.isnan(_np(o["top_logp"])[r]).all()
        assert o["top_tokens"][r].tolist() == [-1] * 4
    keep = [0, 5]
    _check(z[keep], tokens[keep], {k: v[keep] for k, v in o.items()})
    assert int(status) == 0


@pytest.mark.parametrize("classes", [12, 3000, 40000])
def test_rows_that_are_not_valid(classes):
    z = _logits(5, classes, BF16, 10)
    legal = torch.tensor([classes, 3, classes + 1, -1, 0], dtype=I32, device=dev())
    tokens = torch.tensor([0, 3, 0, 0, 0], dtype=I32, device=dev())
    status = torch.zeros(1, dtype=I32, device=dev())
    o = _forward(z, tokens, legal, top=2, status=status)
    grad = torch.full_like(z, 7.0)
    P.dora_token_logprob_grad(z, tokens, o["norm"], grad, dlogp=torch.ones(5, device=dev()),
                              legal=legal, status=status)
    torch.cuda.synchronize()
    assert int(status) == 5
    for r in (1, 2, 3, 4):
        assert np.isnan(_np(o["logp"])[r]) and np.isnan(_np(o["norm"])[r]).all()
        assert o["top_tokens"][r].tolist() == [-1, -1] and np.isnan(_np(grad)[r]).all()
    assert np.isfinite(_np(grad)[0]).all() and np.isfinite(_np(o["logp"])[0])


def _grad_check(z, tokens, legal, temperature, dl, dh, got, o, flush=0.0):
    zz, dtype = _np(z), z.dtype
    tk = None if tokens is None else tokens.cpu().numpy()
    lg = None if legal is None else legal.cpu().numpy()
    dln, dhn = (None if t is None else _np(t) for t in (dl, dh))
    ref = O.token_logprob_grad(zz, tk, dln, dhn, lg, temperature)
    f = O.token_logprob(zz, tk, lg, temperature)
    m, ls, h = f["norm"][:, :1], f["norm"][:, 1:], f["entropy"][:, None]
    n = zz.shape[1]
    with np.errstate(invalid="ignore", over="ignore"):
        d = np.where(np.isfinite(zz - m), np.abs(zz - m), 0.0) / temperature
        p = np.where(np.isfinite(zz), np.exp(np.minimum((zz - m) / temperature - ls, 0)), 0.0)
    mean_d = (p * d).sum(1, keepdims=True)
    e = (n / 512 + 24) * 2.0 ** -24 + 2.0 ** -22 * (4 + mean_d + d + np.abs(ls))
    size = np.zeros_like(zz)
    if dln is not None:
        size += np.abs(dln)[:, None] * p
    if dhn is not None:
        size += np.abs(dhn)[:, None] * p * (d + np.abs(ls) + np.abs(h) + 1) * 2
    if dln is not None:
        rows = np.flatnonzero(tk >= 0)
        size[rows, tk[rows]] += np.abs(dln)[rows] * 0.5
    # flush: probabilities that 32 bits hold as 0
    size_0 = (0 if dln is None else np.abs(dln)[:, None]) + (
        0 if dhn is None else np.abs(dhn)[:, None] * (100 + np.abs(ls) + np.abs(h)))
    r, a = ROUND[dtype]
    a = a + flush * size_0 / temperature
    tol = r * np.abs(ref) + a + (1 + r) * e * size / temperature
    assert np.all(np.abs(_np(got) - ref) <= tol), np.max(np.abs(_np(got) - ref) / tol)


@pytest.mark.parametrize("rows,classes", SIZES)
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("what", ["logp", "both", "entropy"])
def test_gradient(rows, classes, dtype, what):
    pad, shift = (0, 0) if what == "both" else (3, 1)
    temperature = 1.3 if what == "both" else 1.0
    z = _logits(rows, classes, dtype, rows + 2 * classes, pad, shift)
    g = torch.Generator(device=dev()).manual_seed(classes)
    tokens = torch.randint(0, classes, (rows,), generator=g, device=dev(), dtype=I32)
    legal = None
    if what == "both" and rows > 2:
        legal = torch.randint(1, classes + 1, (rows,), generator=g, device=dev(), dtype=I32)
        tokens = (tokens % legal).to(I32)
        tokens[1] = -1
    o = _forward(z, tokens, legal, temperature)
    dl = torch.randn(rows, generator=g, device=dev()) if what != "entropy" else None
    dh = torch.randn(rows, generator=g, device=dev()) * 0.3 if what != "logp" else None
    # a buffer whose other elements keep their values, at another alignment than the logits'
    for lie in (shift, shift + 1):
        ld = classes + pad
        flat = torch.full((lie + rows * ld + 9,), 7.0, dtype=dtype, device=dev())
        grad = flat[lie:lie + rows * ld].view(rows, ld)[:, :classes]
        P.dora_token_logprob_grad(z, tokens, o["norm"], grad, dlogp=dl, dentropy=dh,
                                  entropy=o["entropy"], legal=legal, temperature=temperature)
        torch.cuda.synchronize()
        zz = z.clone()
        if legal is not None:
            zz[torch.arange(classes, device=dev()) >= legal[:, None]] = float("-inf")
        _grad_check(zz, tokens, legal, temperature, dl, dh, grad, o)
        rest = flat.clone()
        rest[lie:lie + rows * ld].view(rows, ld)[:, :classes] = 7.0
        assert bool((rest == 7.0).all())
    same = grad.clone()
    P.dora_token_logprob_grad(z, tokens, o["norm"], z, dlogp=dl, dentropy=dh,
                              entropy=o["entropy"], legal=legal, temperature=temperature)
    torch.cuda.synchronize()
    assert torch.equal(z, same)                    # over the logits: the same bits


def test_gradient_is_the_difference():
    z = _logits(4, 50, F32, 12, scale=1.0)
    tokens = torch.tensor([3, 49, 0, -1], dtype=I32, device=dev())
    dl, dh = torch.tensor([1., -2., .5, 3.], device=dev()), torch.tensor([.3, .1, -1., 2.],
                                                                        device=dev())
    o = _forward(z, tokens, temperature=0.8)
    grad = torch.empty_like(z)
    P.dora_token_logprob_grad(z, tokens, o["norm"], grad, dlogp=dl, dentropy=dh,
                              entropy=o["entropy"], temperature=0.8)
    h = 2.0 ** -6
    for j in (0, 3, 17, 49):
        up, down = z.clone(), z.clone()
        up[:, j] += h
        down[:, j] -= h
        a, b = _forward(up, tokens, temperature=0.8), _forward(down, tokens, temperature=0.8)
        slope = (dl * (a["logp"] - b["logp"]) + dh * (a["entropy"] - b["entropy"])) / (2 * h)
        # third derivatives times h^2 / 6 (each below 4 (|dl| + 8 |dh|) / T^3), and fp32 values
        # of up to 5 over 2 h
        tol = (dl.abs() + 8 * dh.abs()) * (h * h * 4 / 0.5 / 6 + 8e-6 / h)
        assert bool(((slope - grad[:, j]).abs() <= tol).all())


@pytest.mark.parametrize("classes", [20, 900, 6000, 40000])
def test_gradients_of_masked_logits_are_zero(classes):
    z = _logits(3, classes, F32, 13)
    z[0, 1:] = float("-inf")
    z[1, ::2] = torch.finfo(F32).min
    z[2, ::3] = float("-inf")
    tokens = torch.tensor([0, 1, 1], dtype=I32, device=dev())
    o = _forward(z, tokens)
    one = torch.ones(3, device=dev())
    grad = torch.empty_like(z)
    P.dora_token_logprob_grad(z, tokens, o["norm"], grad, dlogp=one, dentropy=one,
                              entropy=o["entropy"])
    torch.cuda.synchronize()
    assert not grad[0].any() and not grad[1, ::2].any() and not grad[2, ::3].any()
    assert bool(torch.isfinite(grad).all())


@pytest.mark.parametrize("rows,classes", [(300, 96), (40, 3000), (2, 60000)])
def test_same_bits_streams_and_graphs(rows, classes):
    z = _logits(rows, classes, BF16, 14, 1)
    tokens = torch.randint(0, classes, (rows,), device=dev(), dtype=I32)
    first = _forward(z, tokens, top=8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    second = _forward(z, tokens, top=8, stream=side)
    side.synchronize()
    dl = torch.ones(rows, device=dev())
    grads = [torch.empty_strided(z.shape, z.stride(), dtype=z.dtype, device=dev()).zero_()
             for _ in range(2)]
    P.dora_token_logprob_grad(z, tokens, first["norm"], grads[0], dlogp=dl)
    third = {k: torch.zeros_like(v) for k, v in first.items()}
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            P.dora_token_logprob(z, tokens, third["logp"], entropy=third["entropy"],
                                 norm=third["norm"], top_logp=third["top_logp"],
                                 top_tokens=third["top_tokens"])
            P.dora_token_logprob_grad(z, tokens, third["norm"], grads[1], dlogp=dl)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    for k, v in first.items():
        assert torch.equal(v, second[k]) and torch.equal(v, third[k])
    assert torch.equal(grads[0], grads[1])


@pytest.mark.parametrize("classes", [20, 900, 6000, 40000])
@pytest.mark.parametrize("temperature", [1e-18, 1e-6, 1e-3, 30.0, 1e6, 1e18])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_extreme_temperatures(classes, temperature, dtype):
    z = _logits(4, classes, dtype, 16)
    z[0, ::3] = float("-inf")
    z[1, ::2] = torch.finfo(dtype).min
    z[2, 1:5] = z[2, :4].clone()
    legal = torch.tensor([classes, classes, classes, classes - 3], dtype=I32, device=dev())
    tokens = torch.tensor([1, 1, 0, 5], dtype=I32, device=dev())
    o = _forward(z, tokens, legal, temperature, top=3)
    dl = torch.tensor([1.0, -2.0, 0.5, 1.0], device=dev())
    dh = torch.tensor([0.5, 1.0, -1.0, 2.0], device=dev())
    grad = torch.full_like(z, 7.0)
    P.dora_token_logprob_grad(z, tokens, o["norm"], grad, dlogp=dl, dentropy=dh,
                              entropy=o["entropy"], legal=legal, temperature=temperature)
    torch.cuda.synchronize()
    # the temperature itself and one over it are rounded: an exponent is 2^-22 of itself off at most
    t = float(np.float32(temperature))
    _check(z, tokens, o, legal, t)
    assert bool(torch.isfinite(grad).all())
    _grad_check(z, tokens, legal, t, dl, dh, grad, o, flush=2.0 ** -126)


def test_another_current_device_is_refused(monkeypatch):
    z = torch.zeros(4, 6, device=dev())
    tokens, f = torch.zeros(4, dtype=I32, device=dev()), torch.zeros(4, device=dev())
    monkeypatch.setattr(P, "_raw_device", lambda: 1)
    with pytest.raises(ValueError, match="current device"):
        P.dora_token_logprob(z, tokens, f)
    with pytest.raises(ValueError, match="current device"):
        P.dora_token_logprob_grad(z, tokens, torch.zeros(4, 2, device=dev()), z, dlogp=f)


def test_empty_batches_and_refusals():
    z = torch.zeros(0, 5, device=dev())
    none = torch.zeros(0, device=dev())
    P.dora_token_logprob(z, none.int(), none)
    P.dora_token_logprob_grad(z, none.int(), none.view(0, 2), z, dlogp=none)
    z = torch.zeros(4, 6, device=dev())
    tokens, f = torch.zeros(4, dtype=I32, device=dev()), torch.zeros(4, device=dev())
    norm = torch.zeros(4, 2, device=dev())
    bad = [dict(logits=z.t()), dict(logits=z[0]), dict(logits=z.double()), dict(tokens=tokens[:3]),
           dict(tokens=tokens.long()), dict(logp=None), dict(tokens=None), dict(classes=7),
           dict(classes=0), dict(legal=tokens[:2]), dict(entropy=f[:1]), dict(norm=f),
           dict(top_logp=torch.zeros(4, 3, device=dev())),
           dict(top_logp=torch.zeros(3, 3, device=dev()),
                top_tokens=torch.zeros(3, 3, dtype=I32, device=dev())),
           dict(top_logp=torch.zeros(4, 33, device=dev()),
                top_tokens=torch.zeros(4, 33, dtype=I32, device=dev())),
           dict(temperature=0.0), dict(temperature=float("nan")), dict(legal=tokens.cpu())]
    for b in bad:
        a = {"logits": z, "tokens": tokens, "logp": f, **b}
        with pytest.raises((TypeError, ValueError, P.DoraError)):
            P.dora_token_logprob(**a)
    for b in [dict(grad=z[:, :5]), dict(grad=z.half()), dict(norm=norm[:3]), dict(dlogp=None),
              dict(tokens=None), dict(dentropy=f), dict(temperature=-1.0),
              dict(grad=torch.zeros(4, 12, device=dev())[:, ::2])]:
        a = {"logits": z, "tokens": tokens, "norm": norm, "grad": z.clone(), "dlogp": f, **b}
        with pytest.raises((TypeError, ValueError, P.DoraError)):
            P.dora_token_logprob_grad(**a)
    wide = torch.empty(1, 2 ** 32 + 5, dtype=BF16, device=dev())
    wide[:, :8] = 0.0
    with pytest.raises(ValueError):
        P.dora_token_logprob(wide, tokens[:1], f[:1])
    P.dora_token_logprob(wide, tokens[:1], f[:1], classes=4)
    assert abs(float(f[0]) + 1.3862944) < 1e-6


def test_rows_past_32_bits():
    # the last row's logits begin past 2^31 elements
    rows, classes = 70000, 40000
    flat = torch.empty(rows * classes, dtype=BF16, device=dev())
    z = flat.view(rows, classes)
    pick = torch.tensor([0, 35000, 69999], device=dev())
    z[pick] = _logits(3, classes, BF16, 15)
    tokens = torch.full((rows,), -1, dtype=I32, device=dev())
    tokens[pick] = torch.tensor([7, 39999, 123], dtype=I32, device=dev())
    o = _forward(z, tokens, top=4)
    P.dora_token_logprob_grad(z, tokens, o["norm"], z, dlogp=torch.ones(rows, device=dev()))
    torch.cuda.synchronize()
    ref = _logits(3, classes, BF16, 15)
    _check(ref, tokens[pick], {k: v[pick] for k, v in o.items()})
    _grad_check(ref, tokens[pick], None, 1.0, torch.ones(3, device=dev()), None, z[pick], o)
    assert not z[1].any() and not z[69998].any()
