"""GPU parity of the gradient norm, clipping and Adam over tensor lists, against
the fp64 oracle.

Bounds.  A norm is one fp32 rounding of a 64-bit sum whose terms carry a few
2^-24 each: 1e-6.  A clipped gradient is one product of two fp32 values (2^-23),
rounded once more in 16 bits (2^-9 and 2^-12).  Adam's moments are one product
and one fused sum: 2^-22 of their larger term; the update a handful of fp32
operations: 1e-6 of it, and the weight one rounding."""
import numpy as np
import pytest
import torch

import __graft_entry__ as G
import oracle as O
import paper_2609_34325_gb300 as P
from helpers import dev

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
ROUND = {BF16: (2.0 ** -8, 0.0), F16: (2.0 ** -11, 2.0 ** -24), F32: (2.0 ** -23, 0.0)}
SIZES = [1, 0, 3, 7, 8, 1023, 1024, 1025, 2047, 4096, 5000, 0, 100003, 64]


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    G.build()
    P.load_library()
    torch.cuda.set_device(0)


def _tensors(sizes, dtypes, seed, scale=1.0, shift=0):
    """Tensors of these sizes, types in turn; with shift, views that start so many
    elements into their storage."""
    g = torch.Generator(device=dev()).manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        t = torch.randn(n + shift, generator=g, device=dev()) * scale
        out.append(t.to(dtypes[i % len(dtypes)])[shift:])
    return out


def _np(t):
    return t.double().cpu().numpy()


def _norm(ts, max_norm=float("inf")):
    out = torch.full((2,), 7.0, device=dev())
    P.dora_grad_norm(P.ParamList(ts), max_norm, out)
    torch.cuda.synchronize()
    return out.cpu().numpy().astype(np.float64)


MIXES = [(F32,), (BF16,), (F16,), (F32, BF16, F16)]


@pytest.mark.parametrize("dtypes", MIXES)
@pytest.mark.parametrize("shift", [0, 1, 3])
@pytest.mark.parametrize("sizes", [SIZES, [1], [0], [0, 0, 5], [3000001], [17] * 500,
                                   [2000] * 3 + [0] * 7])
def test_grad_norm(sizes, dtypes, shift):
    ts = _tensors(sizes, dtypes, len(sizes) + shift, 0.1, shift)
    ref, f = O.grad_norm([_np(t) for t in ts], 0.5)
    got = _norm(ts, 0.5)
    assert abs(got[0] - ref) <= 1e-6 * ref and abs(got[1] - f) <= 1e-6 * f


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e-20, 1e15, 1e25, 1e34])
def test_grad_norm_of_extreme_values(scale):
    # squares leave the range of fp32 on both sides; a few plain values among them
    ts = _tensors([5000, 33, 70000], (F32,), 3, scale)
    ref, _ = O.grad_norm([_np(t) for t in ts], 1.0)
    assert abs(_norm(ts)[0] - ref) <= 1e-6 * ref
    ts.append(_tensors([4000], (BF16,), 4)[0])
    ref, _ = O.grad_norm([_np(t) for t in ts], 1.0)
    assert abs(_norm(ts)[0] - ref) <= 1e-6 * ref


def test_grad_norm_zero_and_not_finite():
    z = [torch.zeros(5000, device=dev()), torch.zeros(9, device=dev(), dtype=BF16)]
    assert _norm(z, 1.0).tolist() == [0.0, 1.0]
    for value in (np.inf, -np.inf, np.nan):
        for n, at in ((5000, 4321), (3, 2), (70001, 70000)):
            ts = _tensors([100, n], (F32, BF16), 5)
            ts[1][at] = value
            got = _norm(ts, 1.0)
            assert not np.isfinite(got[0]) and got[1] == 1.0
    assert _norm(_tensors([4000], (F32,), 6), 0.0)[1] == 0.0


def test_grad_norm_same_bits_streams_and_graphs():
    ts = _tensors([300001, 77, 123456], (F32, BF16), 7)
    lst = P.ParamList(ts)
    out = [torch.zeros(2, device=dev()) for _ in range(3)]
    P.dora_grad_norm(lst, 1.0, out[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    P.dora_grad_norm(lst, 1.0, out[1], stream=side)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            P.dora_grad_norm(lst, 1.0, out[2])
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[2])


@pytest.mark.parametrize("dtypes", MIXES)
@pytest.mark.parametrize("shift,out_shift", [(0, 0), (1, 1), (0, 1)])
@pytest.mark.parametrize("max_norm", [0.5, 1e6])
def test_clip_grads(dtypes, shift, out_shift, max_norm):
    ts = _tensors(SIZES + [400000], dtypes, 11, 0.3, shift)
    before = [_np(t) for t in ts]
    norm, f = O.grad_norm(before, max_norm)
    to = [t.clone() for t in _tensors([t.numel() for t in ts], dtypes, 12, 1.0, 0)]
    to = [torch.full((t.numel() + out_shift,), 7.0, dtype=t.dtype, device=dev())[out_shift:]
          for t in ts]
    out = torch.zeros(2, device=dev())
    P.dora_clip_grads(P.ParamList(ts, clipped=to), max_norm, out)
    torch.cuda.synchronize()
    assert abs(float(out[0]) - norm) <= 1e-6 * norm
    for t, b, c in zip(ts, before, to):
        assert np.array_equal(_np(t), b)                   # the gradients are kept
        r, a = ROUND[t.dtype]
        assert np.all(np.abs(_np(c) - f * b) <= (r + 1e-6) * np.abs(f * b) + a)
        if f == 1.0:
            assert np.array_equal(_np(c), b)
    P.dora_clip_grads(P.ParamList(ts), max_norm, out)      # in place: the same bits
    torch.cuda.synchronize()
    for t, c in zip(ts, to):
        assert torch.equal(t, c)


def test_clip_grads_with_a_norm_that_is_not_finite():
    for value in (np.inf, np.nan):
        ts = _tensors([5000, 70000], (F32, BF16), 13)
        ts[0][77] = value
        before = [t.clone() for t in ts]
        to = [torch.zeros_like(t) for t in ts]
        out = torch.zeros(2, device=dev())
        P.dora_clip_grads(P.ParamList(ts, clipped=to), 0.1, out)
        P.dora_clip_grads(P.ParamList(ts), 0.1, out)
        torch.cuda.synchronize()
        for t, b, c in zip(ts, before, to):
            assert torch.equal(t.nan_to_num(1e9), b.nan_to_num(1e9))
            assert torch.equal(c.nan_to_num(1e9), b.nan_to_num(1e9))


def _adam_inputs(sizes, pt, gt, seed, shift=0):
    g = _tensors(sizes, (gt,), seed, 1e-2, shift)
    p = _tensors(sizes, (pt,), seed + 1, 0.05, shift)
    m = _tensors(sizes, (F32,), seed + 2, 1e-3, shift)
    v = [t.square() for t in _tensors([n + shift for n in sizes], (F32,), seed + 3, 1e-2)]
    return g, p, m, [t[shift:] for t in v]


def _state_step(state):
    return int(state[:8].view(torch.int64).item())


@pytest.mark.parametrize("pt", [F32, BF16, F16])
@pytest.mark.parametrize("gt", [F32, BF16, F16])
@pytest.mark.parametrize("shift", [0, 1, 2])
def test_adam_steps(pt, gt, shift):
    sizes = SIZES + [30011]
    g, p, m, v = _adam_inputs(sizes, pt, gt, 21, shift)
    copies = [torch.zeros(t.numel() + shift, dtype=BF16, device=dev())[shift:] for t in p]
    state = P.alloc_adam_state(dev())
    lst = P.ParamList(g, params=p, exp_avg=m, exp_avg_sq=v, copies=copies)
    hp = dict(beta1=0.9, beta2=0.99, eps=1e-6, weight_decay=0.1)
    norm = torch.zeros(2, device=dev())
    r, a = ROUND[pt]
    for step in range(1, 4):
        ref = []
        n, f = O.grad_norm([_np(t) for t in g], 0.2)
        for i in range(len(p)):
            ref.append(O.adam_step(_np(p[i]), _np(m[i]), _np(v[i]), _np(g[i]), step, 1e-2, 0.9,
                                   0.99, 1e-6, 0.1, f if step > 1 else 1.0))
        old = [_np(t) for t in p]
        old_m, old_v = [_np(t) for t in m], [_np(t) for t in v]
        if step > 1:                                       # the first without clipping
            P.dora_grad_norm(lst, 0.2, norm)
        P.dora_adam_step(lst, state, 1e-2, clip=norm if step > 1 else None, **hp)
        torch.cuda.synchronize()
        assert _state_step(state) == step
        for i in range(len(p)):
            pr, mr, vr = ref[i]
            gi = np.abs(_np(g[i]))
            assert np.all(np.abs(_np(m[i]) - mr) <= 2.0 ** -21 * (np.abs(old_m[i]) + gi))
            assert np.all(np.abs(_np(v[i]) - vr) <= 2.0 ** -20 * (old_v[i] + gi * gi))
            # the update m / sqrt(v) carries its terms' errors where m nearly cancels
            upd = 1e-2 / (1 - 0.9 ** step) * (np.abs(old_m[i]) + gi) / (
                np.sqrt(vr / (1 - 0.99 ** step)) + 1e-6)
            tol = 4e-6 * upd + (r + 2.0 ** -22) * np.abs(pr) + a
            assert np.all(np.abs(_np(p[i]) - pr) <= tol + 1e-9)
            want = _np(p[i].to(BF16)) if pt == F32 else pr
            assert np.all(np.abs(_np(copies[i]) - want) <= (0 if pt == F32 else
                                                            2.0 ** -8 * np.abs(want) + tol))
            assert pr.size == 0 or not np.array_equal(_np(p[i]), old[i])


@pytest.mark.parametrize("shifts", [(1, 0, 0, 0), (0, 2, 1, 1), (3, 3, 3, 1), (0, 0, 1, 3)])
def test_adam_on_buffers_that_lie_differently(shifts):
    # gradients, weights and moments each so many elements into their storage
    sizes = [1, 3, 5, 1027, 4099, 20001]
    g = _tensors(sizes, (BF16,), 61, 1e-2, shifts[0])
    p = _tensors(sizes, (F32,), 62, 0.05, shifts[1])
    m = _tensors(sizes, (F32,), 63, 1e-3, shifts[2])
    v = [t.square() for t in _tensors([n + shifts[3] for n in sizes], (F32,), 64, 1e-2)]
    v = [t[shifts[3]:] for t in v]
    ref = [O.adam_step(_np(p[i]), _np(m[i]), _np(v[i]), _np(g[i]), 1, 1e-2, 0.9, 0.999, 1e-8, 0.0)
           for i in range(len(p))]
    top = [1e-1 * (np.abs(_np(m[i])) + np.abs(_np(g[i]))) / (np.sqrt(ref[i][2] / 1e-3) + 1e-8)
           for i in range(len(p))]
    P.dora_adam_step(P.ParamList(g, params=p, exp_avg=m, exp_avg_sq=v), P.alloc_adam_state(dev()),
                     1e-2)
    torch.cuda.synchronize()
    for i in range(len(p)):
        pr, mr, vr = ref[i]
        assert np.all(np.abs(_np(m[i]) - mr) <= 2.0 ** -21 * (np.abs(mr) + np.abs(_np(g[i]))) + 1e-9)
        assert np.all(np.abs(_np(v[i]) - vr) <= 2.0 ** -20 * vr + 1e-12)
        assert np.all(np.abs(_np(p[i]) - pr) <= 4e-6 * top[i] + 2.0 ** -21 * np.abs(pr) + 1e-9)


def test_adam_skips_a_norm_that_is_not_finite():
    g, p, m, v = _adam_inputs([3000, 5], F32, F32, 31)
    state = P.alloc_adam_state(dev(), step=7)
    lst = P.ParamList(g, params=p, exp_avg=m, exp_avg_sq=v)
    norm = torch.zeros(2, device=dev())
    before = [t.clone() for t in p + m + v]
    g[0][5] = np.inf
    P.dora_grad_norm(lst, 1.0, norm)
    P.dora_adam_step(lst, state, 1e-3, clip=norm)
    torch.cuda.synchronize()
    assert _state_step(state) == 7
    for t, b in zip(p + m + v, before):
        assert torch.equal(t, b)
    g[0][5] = 0.0                                          # and goes on with the next
    P.dora_grad_norm(lst, 1.0, norm)
    P.dora_adam_step(lst, state, 1e-3, clip=norm)
    torch.cuda.synchronize()
    assert _state_step(state) == 8 and not torch.equal(p[0], before[0])


def test_adam_resumes_and_replays():
    # five steps; three, a state made anew, two; and five replays of one captured step
    runs = []
    for how in range(3):
        g, p, m, v = _adam_inputs([2500, 40], F32, BF16, 41)
        lst = P.ParamList(g, params=p, exp_avg=m, exp_avg_sq=v)
        state = P.alloc_adam_state(dev())
        if how == 2:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.stream(side):
                with torch.cuda.graph(graph, stream=side):
                    P.dora_adam_step(lst, state, 1e-2)
            for _ in range(5):
                graph.replay()
        else:
            for i in range(5):
                if how == 1 and i == 3:
                    state = P.alloc_adam_state(dev(), step=3)
                P.dora_adam_step(lst, state, 1e-2)
        torch.cuda.synchronize()
        assert _state_step(state) == 5
        runs.append(torch.cat([t.float() for t in p + m + v]))
    assert torch.equal(runs[0], runs[2])
    assert torch.allclose(runs[0], runs[1], rtol=1e-6, atol=0)


def test_adam_list_without_weights_is_refused():
    g, p, m, v = _adam_inputs([100], F32, F32, 51)
    with pytest.raises(P.DoraError):
        P.dora_adam_step(P.ParamList(g), P.alloc_adam_state(dev()), 1e-3)
    with pytest.raises(TypeError):
        P.ParamList(g, params=p, exp_avg=[m[0].to(BF16)], exp_avg_sq=v)
    with pytest.raises(ValueError):
        P.ParamList(g, params=[p[0][:50]], exp_avg=m, exp_avg_sq=v)
    with pytest.raises(TypeError):
        P.ParamList([g[0][::2]])
    with pytest.raises(TypeError):
        P.dora_grad_norm(g, 1.0, torch.zeros(2, device=dev()))


def test_lists_past_32_bits():
    # one gradient of 2.2e9 elements, its end past 2^31
    n = 2_200_000_000
    g = torch.zeros(n, dtype=BF16, device=dev())
    g[-5:] = 3.0
    g[0] = 6.0
    out = torch.zeros(2, device=dev())
    P.dora_clip_grads(P.ParamList([g]), 4.5, out)
    torch.cuda.synchronize()
    assert out.tolist() == [9.0, 0.5]
    assert g[-6:].tolist() == [0.0] + [1.5] * 5 and float(g[0]) == 3.0
