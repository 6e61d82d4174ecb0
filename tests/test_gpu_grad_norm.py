"""am_grad_norm and am_clip_grads against the same sums in 64 bits.

Bounds: squares are summed in fp64 (relative error below n 2^-53, far below an fp32 unit), norm and factor are rounded once to
fp32: 2^-24 of themselves.  A clipped gradient is a product of two fp32 numbers rounded once, with a factor that may be off by 2^-24:
2^-23 in fp32; in bf16 2^-8 of itself and a little.  Packing without scaling is exact, or one rounding to bf16."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


def _grads(R, sizes, types, seed, scale=1e-3):
    gen = torch.Generator().manual_seed(seed)
    return [[(torch.randn(n, generator=gen) * scale).to(t).cuda() for n, t in zip(sizes, types)] for _ in range(R)]


def _want(grads, max_norm):
    norm = torch.tensor([math.sqrt(sum(float((g.double() ** 2).sum()) for g in gs)) for gs in grads], dtype=torch.float64)
    return norm, torch.where(norm <= max_norm, torch.ones_like(norm), max_norm / norm)


def _check_norms(got, want):
    for g, w in zip(got, want):
        assert g.dtype == F and g.shape == w.shape
        assert bool(((g.double().cpu() - w).abs() <= 2.0 ** -24 * 1.001 * w).all()), (g, w)


def _check_scaled(got, grads, factor, unit):
    for o, gs, f in zip(got, grads, factor):
        want = torch.cat([g.double().reshape(-1) for g in gs]) * float(f) if gs else torch.empty(0, dtype=torch.float64, device="cuda")
        assert bool(((o.double() - want).abs() <= unit * want.abs() + 1e-42).all())


SHAPES = [([1], [F]), ([1], [BF]), ([0, 5, 0], [F, BF, BF]), ([7, 8192, 8193, 1, 3], [BF] * 5), ([100_003, 2, 16384], [F, BF, F]), ([13] * 130, [F, BF] * 65),
          ([1_000_001, 999], [BF, BF])]


@pytest.mark.parametrize("sizes,types", SHAPES)
@pytest.mark.parametrize("R", [1, 3])
@pytest.mark.parametrize("out", [None, F, BF])
def test_norm_and_packing(amlib, sizes, types, R, out):
    print("grad_norm", sizes[:6], R, out, flush=True)
    grads = _grads(R, sizes, types, 1)
    norm, _ = _want(grads, 1.0)
    max_norm = float(norm.mean())
    flat = None if out is None else [torch.full((sum(sizes),), 7.0, dtype=out, device="cuda") for _ in range(R)]
    got = amlib.grad_norm(grads, max_norm, out=flat)
    _check_norms(got, _want(grads, max_norm))
    if flat:
        for o, gs in zip(flat, grads):
            assert torch.equal(o, torch.cat([g.to(out) for g in gs]))


@pytest.mark.parametrize("sizes,types", SHAPES)
@pytest.mark.parametrize("R", [1, 3])
@pytest.mark.parametrize("out", [None, F, BF])
def test_clipping(amlib, sizes, types, R, out):
    print("clip_grads", sizes[:6], R, out, flush=True)
    grads = _grads(R, sizes, types, 2)
    before = [[g.clone() for g in gs] for gs in grads]
    max_norm = 0.5 * float(_want(grads, 1.0)[0].min())
    flat = None if out is None else [torch.full((sum(sizes) + 3,), 7.0, dtype=out, device="cuda") for _ in range(R)]
    got = amlib.clip_grads(grads, max_norm, out=None if out is None else [f[1:1 + sum(sizes)] for f in flat])
    want = _want(before, max_norm)
    _check_norms(got, want)
    if out is None:
        for i in range(R):
            for g, b in zip(grads[i], before[i]):
                _check_scaled([g.reshape(-1)], [[b]], [want[1][i]], 2.0 ** -22 if g.dtype == F else 2.0 ** -8 * 1.001)
    else:
        assert all(torch.equal(g, b) for gs, bs in zip(grads, before) for g, b in zip(gs, bs))
        _check_scaled([f[1:-2] for f in flat], before, want[1], 2.0 ** -22 if out == F else 2.0 ** -8 * 1.001)
        assert all(bool((f[[0, -2, -1]] == 7).all()) for f in flat)


def test_a_norm_within_the_bound_changes_nothing(amlib):
    grads = _grads(2, [1001, 64], [F, BF], 3)
    before = [[g.clone() for g in gs] for gs in grads]
    norm, factor = amlib.clip_grads(grads, 1e6)
    assert bool((factor == 1).all()) and all(torch.equal(a, b) for x, y in zip(grads, before) for a, b in zip(x, y))
    assert bool((amlib.grad_norm(grads)[1] == 1).all())
    zero = [[torch.zeros(100, device="cuda")]]
    norm, factor = amlib.clip_grads(zero, 0.0)
    assert float(norm) == 0 and float(factor) == 1


def test_range_of_the_squares(amlib):
    """Squares that fp32 has no room for."""
    for scale in (1e-30, 1e25):
        g = [[torch.full((4096,), scale, device="cuda")]]
        norm, factor = amlib.grad_norm(g, scale)
        assert abs(float(norm) / (64 * scale) - 1) < 1e-6 and abs(float(factor) * 64 - 1) < 1e-6


def test_values_that_are_not_finite(amlib):
    for bad in (float("nan"), float("inf")):
        grads = _grads(2, [50, 3000], [F, BF], 4)
        grads[1][1][2999] = bad
        norm, factor = amlib.grad_norm(grads, 1e-3)
        assert math.isfinite(float(norm[0])) and float(factor[0]) < 1
        if math.isnan(bad):
            assert math.isnan(float(norm[1])) and math.isnan(float(factor[1]))
        else:
            assert math.isinf(float(norm[1])) and float(factor[1]) == 0


def test_many_replicas_and_many_tensors(amlib):
    """More pointers than one launch takes."""
    grads = _grads(32, [100] * 70, [F] * 70, 5)
    flat = [torch.empty(7000, device="cuda") for _ in range(32)]
    got = amlib.grad_norm(grads, 0.01, out=flat)
    _check_norms(got, _want(grads, 0.01))
    assert all(torch.equal(o, torch.cat(gs)) for o, gs in zip(flat, grads))


def test_no_tensors(amlib):
    out = [torch.empty(0, device="cuda")]
    norm, factor = amlib.grad_norm([[]], 1.0, out=out)
    assert float(norm) == 0 and float(factor) == 1


def test_the_factors_are_what_the_step_takes(amlib):
    """Packing with factors given to step_scaled against clipping first, on a stage: the same weights to rounding (the step's factor
    multiplies in fp64, the clipped gradient was rounded: 2^-23 of an update of at most lr)."""
    am = amlib
    sizes, lr = [300, 4000, 77], 3e-4
    n = sum(sizes)
    w0 = torch.randn(n, device="cuda") * 0.02
    grads = _grads(2, sizes, [F] * 3, 6)
    max_norm = 0.3 * float(am.grad_norm(grads)[0].min())
    a, b = (am.init_state(am.make_config(n, 2, delay=1, fraction=0.1, optimizer=am.OPT_SGD, beta1=0.9), w0) for _ in range(2))
    flat = [torch.empty(n, device="cuda") for _ in range(2)]
    _, factor = am.grad_norm(grads, max_norm, out=flat)
    a.step_scaled(1, flat, lr, 0.5, 1.0, factor)
    am.clip_grads(grads, max_norm, out=flat)
    b.step(1, flat, lr, 0.5)
    for x, y in zip(a.w, b.w):
        assert bool(((x - y).abs() <= 2.0 ** -23 * (w0.abs() + lr)).all())


def test_in_a_graph(amlib):
    am = amlib
    grads = _grads(2, [5000, 321], [BF, F], 7)
    flat = [torch.empty(5321, device="cuda") for _ in range(2)]
    am.clip_grads(grads, 0.01, out=flat)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm, factor = am.clip_grads(grads, 0.01, out=flat)
    for k in range(3):
        for gs, new in zip(grads, _grads(2, [5000, 321], [BF, F], 20 + k)):
            for g, x in zip(gs, new):
                g.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (norm, factor, *flat)]
        n, f = am.clip_grads(grads, 0.01, out=flat)
        assert all(torch.equal(x, y) for x, y in zip(got, (n, f, *flat)))
