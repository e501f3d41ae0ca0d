"""GPU parity of token log-probabilities where there are many rows: the kernels for 4 and 8 rows
an SM and more, whose rows a warp, 64 or 128 threads hold.

A batch repeats 16 rows, whose copies have the same alignment (16 pitches are a multiple of
16 bytes): the first 16 are compared with the fp64 oracle, the others with them, bit by bit.

Bounds.  A thread adds n / threads exponentials in two sums, n / (2 threads) additions each of
2^-24 of what it adds to at most, each exponential 2^-22 of itself off, its exponent 2^-22 of
|d| / T; sums over lanes and warps follow.  So s is off by
e_s = (n / (2 threads) + 24) 2^-24 + 2^-22 (1 + E|d| / T), ln s by that; l adds 2^-22 |d_a| / T,
the entropy the same errors of t / (T s)."""
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
DISTINCT = 16


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    G.build()
    P.load_library()
    torch.cuda.set_device(0)


def _np(t):
    return t.detach().double().cpu().numpy()


# (rows from the SMs, granules of 16 bytes a row may touch, threads a row)
KINDS = {"warp": (lambda sms: 8 * sms + 1, 250, 32),          # 129 to 256 granules
         "64 at the border": (lambda sms: 8 * sms, 250, 64),
         "64": (lambda sms: 8 * sms + 1, 700, 64),
         "128": (lambda sms: 4 * sms + 1, 700, 128),
         "128 short": (lambda sms: 4 * sms, 140, 128)}


def _sizes(kind, dtype):
    rows, granules, threads = KINDS[kind]
    e = 4 if dtype == F32 else 8
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    return rows(sms), granules * e - 2 * e + 3, threads      # odd numbers of classes


def _rows(distinct, rows, pad=0, shift=0):
    """Rows that repeat the distinct ones, in a buffer of NaN: `pad` apart, `shift` elements in."""
    classes = distinct.shape[1]
    ld = classes + pad
    flat = torch.full((shift + rows * ld + 16,), float("nan"), dtype=distinct.dtype, device=dev())
    z = flat[shift:shift + rows * ld].view(rows, ld)[:, :classes]
    z.copy_(distinct.repeat((rows + DISTINCT - 1) // DISTINCT, 1)[:rows])
    return z


def _repeat(t, rows):
    return t.repeat((rows + DISTINCT - 1) // DISTINCT)[:rows].contiguous()


def _noise(classes, dtype, seed, scale=2.5, step=0.0):
    g = torch.Generator(device=dev()).manual_seed(seed)
    v = torch.randn(DISTINCT, classes, generator=g, device=dev()) * scale
    return (torch.round(v / step) * step if step else v).to(dtype)


def _run(z, tokens, legal=None, temperature=1.0, top=0, status=None):
    rows = z.shape[0]
    o = {"logp": torch.full((rows,), 7.0, device=dev()),
         "entropy": torch.full((rows,), 7.0, device=dev()),
         "norm": torch.full((rows, 2), 7.0, device=dev()),
         "top_logp": torch.full((rows, top), 7.0, device=dev()),
         "top_tokens": torch.full((rows, top), 7, dtype=I32, device=dev())}
    P.dora_token_logprob(z, tokens, o["logp"], legal=legal, temperature=temperature,
                         entropy=o["entropy"], norm=o["norm"],
                         top_logp=o["top_logp"] if top else None,
                         top_tokens=o["top_tokens"] if top else None, status=status)
    torch.cuda.synchronize()
    for k, v in o.items():                      # copies of a row: the same bits
        first = v[:DISTINCT]
        bits = v.view(torch.int32) if v.dtype == F32 else v
        want = first.view(torch.int32) if v.dtype == F32 else first
        for r in range(0, rows, DISTINCT):
            some = min(DISTINCT, rows - r)
            assert torch.equal(bits[r:r + some], want[:some]), (k, r)
    return {k: v[:DISTINCT] for k, v in o.items()}


def _check(z, tokens, o, threads, legal=None, temperature=1.0, rows=range(DISTINCT)):
    rows = list(rows)
    zz, tk = _np(z[:DISTINCT][rows]), tokens[:DISTINCT].cpu().numpy()[rows]
    lg = None if legal is None else legal[:DISTINCT].cpu().numpy()[rows]
    got = {k: _np(v)[rows] for k, v in o.items()}
    top = got["top_tokens"].shape[1]
    ref = O.token_logprob(zz, tk, lg, temperature, top)
    n = zz.shape[1]
    with np.errstate(invalid="ignore", divide="ignore"):
        d = np.abs(zz - ref["norm"][:, :1]) / temperature
        d = np.where(np.isfinite(d), d, 0.0)
        p = np.where(np.isneginf(zz), 0.0, np.exp(-d))
    if lg is not None:
        p[np.arange(n) >= lg[:, None]] = 0
    mean_d = (p * d).sum(1) / np.maximum(p.sum(1), 1e-300)
    e_s = (n / (2 * threads) + 24) * 2.0 ** -24 + 2.0 ** -22 * (1 + mean_d)
    tol = e_s + 2.0 ** -22 * (1 + np.abs(ref["norm"][:, 1]))
    takes = (tk >= 0) & (np.ones(len(tk), bool) if lg is None else lg > 0)
    assert np.array_equal(got["norm"][:, 0], ref["norm"][:, 0])
    assert np.all(np.abs(got["norm"][:, 1] - ref["norm"][:, 1]) <= tol)
    assert np.all(np.abs(got["entropy"] - ref["entropy"]) <= tol + 3 * e_s * (1 + mean_d))
    da = d[np.arange(len(tk)), np.where(takes, tk, 0)]
    with np.errstate(invalid="ignore"):
        off = np.abs(got["logp"] - ref["logp"])
    assert np.all((got["logp"] == ref["logp"]) | (off <= tol + 2.0 ** -22 * da))
    assert not got["logp"][~takes].any()
    assert np.array_equal(got["top_tokens"].astype(int), ref["top_tokens"])
    there = ref["top_tokens"] >= 0
    da = np.take_along_axis(d, np.maximum(ref["top_tokens"], 0).astype(int), 1)
    with np.errstate(invalid="ignore"):
        fine = np.abs(got["top_logp"] - ref["top_logp"]) <= tol[:, None] + 2.0 ** -22 * da
    assert np.all(np.where(there, fine, np.isneginf(got["top_logp"])))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("pad,shift,top", [(0, 0, 8), (1, 3, 32), (5, 1, 0)])
def test_forward(kind, dtype, pad, shift, top):
    rows, classes, threads = _sizes(kind, dtype)
    z = _rows(_noise(classes, dtype, 1), rows, pad, shift)
    g = torch.Generator(device=dev()).manual_seed(2)
    tokens = _repeat(torch.randint(0, classes, (DISTINCT,), generator=g, device=dev(), dtype=I32),
                     rows)
    t = 1.0 if pad else 0.7
    _check(z, tokens, _run(z, tokens, temperature=t, top=top), threads, temperature=t)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("top", [8, 32])
def test_legal_prefixes_and_rows_without_a_token(kind, dtype, top):
    rows, classes, threads = _sizes(kind, dtype)
    base = _noise(classes, dtype, 3)
    g = torch.Generator(device=dev()).manual_seed(4)
    legal = torch.randint(1, classes + 1, (DISTINCT,), generator=g, device=dev(), dtype=I32)
    legal[:4] = torch.tensor([0, 1, classes, 2], device=dev())
    tokens = (torch.rand(DISTINCT, generator=g, device=dev()) * legal).to(I32)
    tokens[legal == 0] = -1
    tokens[5::7] = -100
    seen = base.clone()
    for r in range(DISTINCT):
        seen[r, int(legal[r]):] = float("nan")            # not read
        if tokens[r] < 0:
            seen[r] = float("nan")
    z = _rows(seen, rows, 3, 2)
    legal, tokens = _repeat(legal, rows), _repeat(tokens, rows)
    status = torch.zeros(1, dtype=I32, device=dev())
    o = _run(z, tokens, legal, top=top, status=status)
    _check(base, tokens, o, threads, legal)
    assert int(status) == 0


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("step", [0.5, 4.0, 100.0])
@pytest.mark.parametrize("top", [1, 8, 32])
def test_equal_logits_come_by_index(kind, step, top):
    rows, classes, threads = _sizes(kind, BF16)
    base = _noise(classes, BF16, 5, step=step)
    base[2] = -0.0
    base[2, ::3] = 0.0
    z = _rows(base, rows, 1)
    tokens = torch.zeros(rows, dtype=I32, device=dev())
    _check(z, tokens, _run(z, tokens, top=top), threads)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_masked_and_not_finite_rows(kind, dtype):
    rows, classes, threads = _sizes(kind, dtype)
    low = torch.finfo(dtype).min
    base = _noise(classes, dtype, 6)
    base[0] = float("-inf")
    base[0, classes // 2] = 1.0                           # one logit left: certain
    base[1, 1:] = low
    base[2, ::2] = float("-inf")
    base[3] = low                                         # all the same: uniform
    base[4, 3:] = float("-inf")
    base[5, classes - 1] = float("nan")
    base[6, 0] = float("inf")
    base[7] = float("-inf")
    base[8] = float("inf")
    base[9] = torch.linspace(-9, 9, classes, device=dev()).to(dtype)
    base[10] = base[9].flip(0)
    z = _rows(base, rows, 2, 1)
    tokens = torch.ones(DISTINCT, dtype=I32, device=dev())
    tokens[0], tokens[2] = classes // 2, 0
    tokens = _repeat(tokens, rows)
    status = torch.zeros(1, dtype=I32, device=dev())
    o = _run(z, tokens, top=6, status=status)
    for r in (5, 6, 7, 8):
        assert np.isnan(_np(o["logp"])[r]) and np.isnan(_np(o["entropy"])[r])
        assert np.isnan(_np(o["norm"])[r]).all() and np.isnan(_np(o["top_logp"])[r]).all()
        assert o["top_tokens"][r].tolist() == [-1] * 6
    _check(z, tokens, o, threads, rows=[r for r in range(DISTINCT) if not 5 <= r <= 8])
    assert float(o["logp"][0]) == 0.0 and float(o["entropy"][0]) == 0.0
    assert np.isneginf(float(o["logp"][2]))
    assert int(status) == 0


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("temperature", [1e-18, 1e-3, 30.0, 1e18])
def test_extreme_temperatures(kind, temperature):
    rows, classes, threads = _sizes(kind, F32)
    base = _noise(classes, F32, 7)
    base[0, ::3] = float("-inf")
    base[1, ::2] = torch.finfo(F32).min
    z = _rows(base, rows)
    tokens = torch.ones(rows, dtype=I32, device=dev())
    o = _run(z, tokens, temperature=temperature, top=3)
    _check(z, tokens, o, threads, temperature=float(np.float32(temperature)))


@pytest.mark.parametrize("kind", ["64", "128"])
@pytest.mark.parametrize("dtype,step", [(BF16, 0.0), (F32, 0.0), (BF16, 2.0)])
def test_long_rows(kind, dtype, step):
    # several batches of granules to a place of the alternatives' search; with a step many of
    # them are equal
    rows, _, threads = _sizes(kind, dtype)
    classes = 131075
    z = _rows(_noise(classes, dtype, 8, step=step), rows, 2)
    tokens = torch.full((rows,), 7, dtype=I32, device=dev())
    _check(z, tokens, _run(z, tokens, top=32), threads)


def test_tokens_outside_their_rows_are_not_valid():
    for kind in KINDS:
        rows, classes, _ = _sizes(kind, BF16)
        z = _rows(_noise(classes, BF16, 9), rows)
        legal = torch.full((DISTINCT,), classes, dtype=I32, device=dev())
        legal[1:5] = torch.tensor([3, classes + 1, -1, 0], dtype=I32, device=dev())
        tokens = torch.zeros(DISTINCT, dtype=I32, device=dev())
        tokens[1] = 3
        status = torch.zeros(1, dtype=I32, device=dev())
        o = _run(z, _repeat(tokens, rows), _repeat(legal, rows), top=2, status=status)
        assert int(status) == 5
        for r in (1, 2, 3, 4):
            assert np.isnan(_np(o["logp"])[r]) and np.isnan(_np(o["norm"])[r]).all()
            assert o["top_tokens"][r].tolist() == [-1, -1]
        assert np.isfinite(_np(o["logp"])[[0, 5, 15]]).all()


@pytest.mark.parametrize("rows,classes", [(3, 60), (3, 700), (3, 5000), (2, 70000), (1500, 3000)])
def test_logits_further_apart_than_32_bits_hold(rows, classes):
    # -3e38 lies 6e38 below 3e38: with temperature 1e10 6e28, of which a float is 2^-22 off at most
    z = torch.zeros(rows, classes, device=dev())
    z[:, 0], z[:, 1], z[:, 2] = 3e38, -3e38, float("-inf")
    for token, want in ((1, 6e28), (3, 3e28)):
        tokens = torch.full((rows,), token, dtype=I32, device=dev())
        logp, top_logp = torch.zeros(rows, device=dev()), torch.zeros(rows, 32, device=dev())
        top_tokens = torch.zeros(rows, 32, dtype=I32, device=dev())
        P.dora_token_logprob(z, tokens, logp, temperature=1e10, top_logp=top_logp,
                             top_tokens=top_tokens)
        torch.cuda.synchronize()
        assert np.all(np.abs(_np(logp) + want) <= want * 2.0 ** -22)
        assert bool((top_tokens[:, 0] == 0).all()) and not top_logp[:, 0].any()
        assert np.all(np.abs(_np(top_logp[:, 1:]) + 3e28) <= 3e28 * 2.0 ** -22)
