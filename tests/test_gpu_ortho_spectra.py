"""GPU parity of the orthogonalised updates where few directions hold most of a matrix: what
lies beside them is raised by 3.4445 an iteration, and so is every error there.

Bounds.  Operands have 22 bits.  An iteration's four roundings (of X as it is kept, of what
X, F and G go into the products as, the sums' among them) are 2^-22 of X's Frobenius norm at
most, and grow by 3.4445 at most in each iteration that follows:
  4 2^-22 sum_k 3.4445^(4 - k) |X_k| / |X_5|,
with the norms of the iteration itself in 64 bits.  The products' sums are cut off, not rounded, at
each of their 16 values: 3 n 2^-28 of themselves over n of them (half of 2^-23 on average, three
products), of which the iterations make less than four times: 3 (m + n) 2^-26.  Weights of 0, a
rate of 1 and no momentum show the result in 32 bits."""
import numpy as np
import pytest
import torch

import __graft_entry__ as G
import oracle as O
import paper_2609_34325_gb300 as P
from helpers import dev

pytestmark = pytest.mark.gpu

F32 = torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    G.build()
    P.load_library()
    torch.cuda.set_device(0)


def _few_directions(m, n, k, noise, seed, active=None):
    """m x n of k strong directions over noise; active: in so many rows, 0 in the others."""
    rng = np.random.default_rng(seed)
    rows = m if active is None else active
    part = rng.standard_normal((rows, k)) @ rng.standard_normal((k, n)) / k ** 0.5
    part += noise * rng.standard_normal((rows, n))
    x = np.zeros((m, n))
    x[np.sort(rng.permutation(m)[:rows])] = part
    return x.astype(np.float32)


def _bound(x, steps=5):
    m, n = min(x.shape), max(x.shape)
    y = x.astype(np.float64)
    y = y / np.linalg.norm(y)
    a, b, c = O.NS_COEF
    norms = []
    for _ in range(steps):
        norms.append(np.linalg.norm(y))
        gram = y @ y.T if y.shape[0] <= y.shape[1] else y.T @ y
        poly = b * gram + c * gram @ gram
        y = a * y + (poly @ y if y.shape[0] <= y.shape[1] else y @ poly)
    grown = sum(3.4445 ** (steps - 1 - k) * s for k, s in enumerate(norms))
    return 4 * 2.0 ** -22 * grown / np.linalg.norm(y) + 3 * (m + n) * 2.0 ** -26


def _check(xs, steps=5):
    grads = [torch.from_numpy(x).to(dev()) for x in xs]
    params = [torch.zeros_like(g) for g in grads]
    lst = P.MatrixList(grads, params=params, momentum=[torch.zeros_like(g) for g in grads],
                       scales=[1.0] * len(grads))
    P.dora_muon_step(lst, 1.0, momentum=0.0, steps=steps)
    torch.cuda.synchronize()
    for x, p in zip(xs, params):
        ref = O.newton_schulz(x.astype(np.float64), steps)
        off = np.linalg.norm(-p.double().cpu().numpy() - ref) / np.linalg.norm(ref)
        assert off <= _bound(x, steps), (x.shape, off, _bound(x, steps))


# Matrices that a CTA or a cluster holds, each with its transpose.
SMALL = [(33, 33), (33, 300), (40, 40), (64, 512), (64, 787), (65, 65), (65, 600), (96, 128),
         (100, 1100), (128, 128), (128, 768), (128, 2048)]


@pytest.mark.parametrize("shape", SMALL)
@pytest.mark.parametrize("k,noise", [(1, 1e-2), (1, 1e-3), (3, 1e-4), (8, 1e-3)])
def test_small_matrices_of_few_directions(shape, k, noise):
    x = _few_directions(*shape, k, noise, 1)
    _check([x, np.ascontiguousarray(_few_directions(*shape, k, noise, 2).T)])


@pytest.mark.parametrize("shape", SMALL)
@pytest.mark.parametrize("active,noise", [(1, 0.0), (2, 1.0), (2, 3e-3), (4, 3e-3), (16, 1e-2)])
def test_small_matrices_of_few_rows_that_are_not_zero(shape, active, noise):
    x = _few_directions(*shape, 1, noise, 3, active)
    _check([x, np.ascontiguousarray(_few_directions(*shape, 1, noise, 4, active).T)])


@pytest.mark.parametrize("shape", SMALL)
def test_small_matrices_of_noise(shape):
    x = np.random.default_rng(5).standard_normal(shape).astype(np.float32)
    _check([x, np.ascontiguousarray(x.T)])
    _check([x], steps=1)
    _check([x], steps=3)


# Columns go to the CTAs of a cluster by 64, an equal share each, rounded up: nine 64s to four CTAs
# as 3, 3, 3 and 0, eighteen to eight as 3 each to the first six.
@pytest.mark.parametrize("shape", [(64, 520), (100, 520), (20, 576), (1, 513), (128, 1100),
                                   (33, 1344), (128, 1025)])
def test_clusters_whose_last_ctas_have_no_columns(shape):
    x = np.random.default_rng(12).standard_normal(shape).astype(np.float32)
    _check([x, np.ascontiguousarray(x.T)] * 3)
    if shape[0] > 1:
        x = _few_directions(*shape, 1, 1e-3, 13)
        _check([x, np.ascontiguousarray(x.T)], steps=4)


# Matrices whose products are cut into tiles: odd and even numbers of blocks each way, few rows of
# many columns.
LARGE = [(2, 2049), (4, 4096), (8, 4096), (16, 3000), (129, 129), (130, 1100), (200, 300),
         (257, 511), (300, 600), (384, 384), (390, 1000), (640, 700)]


@pytest.mark.parametrize("shape", LARGE)
@pytest.mark.parametrize("k,noise", [(1, 1e-2), (1, 1e-3), (3, 1e-4), (8, 1e-3)])
def test_large_matrices_of_few_directions(shape, k, noise):
    x = _few_directions(*shape, k, noise, 6)
    _check([x, np.ascontiguousarray(_few_directions(*shape, k, noise, 7).T)])


@pytest.mark.parametrize("shape", LARGE)
@pytest.mark.parametrize("active,noise", [(1, 0.0), (2, 1.0), (2, 3e-3)])
def test_large_matrices_of_few_rows_that_are_not_zero(shape, active, noise):
    x = _few_directions(*shape, 1, noise, 8, active)
    _check([x, np.ascontiguousarray(_few_directions(*shape, 1, noise, 9, active).T)])


@pytest.mark.parametrize("shape", LARGE)
@pytest.mark.parametrize("steps", [1, 2, 3, 4, 5])
def test_large_matrices_of_noise(shape, steps):
    x = np.random.default_rng(10).standard_normal(shape).astype(np.float32)
    _check([x, np.ascontiguousarray(x.T)], steps)


def test_matrices_of_few_directions_in_a_list():
    # wide tiles and narrow ones, small matrices beside large ones
    shapes = [(384, 384), (1536, 384), (384, 1152), (64, 787), (2, 2049), (640, 1024)] * 5
    _check([_few_directions(*s, 1 + i % 3, 1e-3, 11 + i) for i, s in enumerate(shapes)])
    _check([_few_directions(1024, 1024, 1, 3e-3, 50)])


# The sums over m, of G X, are cut off beside the strong directions too, where the iterations raise
# what is lost: with larger m more than the term above allows.  The documented bound has m 2^-22
# for them: 3 m / 16 additions, each short of up to 2^-23 of what there is, at random 2^-24 of it,
# together sqrt(3 m / 16) of that, grown by up to 3.4445^4 = 141: 61 2^-24 sqrt(m), below m 2^-22
# from 233 rows on.
@pytest.mark.parametrize("shape", [(2048, 2048), (1024, 9000)])
@pytest.mark.parametrize("noise", [1e-2, 1e-3, 1e-4])
def test_long_sums_hold_the_documented_bound(shape, noise):
    m, n = shape
    g = torch.Generator(device=dev()).manual_seed(60)
    x = torch.randn(m, 1, generator=g, device=dev()) @ torch.randn(1, n, generator=g, device=dev())
    x += noise * torch.randn(m, n, generator=g, device=dev())
    a, b, c = O.NS_COEF
    y = x.double()
    y /= y.norm()
    for _ in range(5):
        gram = y @ y.t()
        y = a * y + (b * gram + c * gram @ gram) @ y
    p = torch.zeros_like(x)
    P.dora_muon_step(P.MatrixList([x], params=[p], momentum=[torch.zeros_like(x)], scales=[1.0]),
                     1.0, momentum=0.0)
    torch.cuda.synchronize()
    assert float((-p.double() - y).norm() / y.norm()) <= 3e-4 + m * 2.0 ** -22 + n * 2.0 ** -26
