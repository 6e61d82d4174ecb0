"""am_linear and am_linear_backward against the same formulas in 64 bits.

Bounds, from the arithmetic: an output is rounded once (half a unit in the last place: at most 2^-8 of its own size with the eight bits of bf16, 2^-24 in fp32), and its sum of
L products is accumulated in fp32 in some order: |error| <= (L + 8) 2^-24 sum |a b| at the very worst; the test allows
sqrt(L) of it times eight.  With an activation dz is rounded to the inputs' type before the products: 2^-8 (bf16) or
2^-24 of sum |dz w| at worst, sqrt(L) of the largest terms in earnest; the sum of squares bounds it.  Activations themselves are good to
2^-20 of max(|z|, 1)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

ACTS = ("NONE", "RELU", "GELU", "GELU_TANH", "SILU")
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def _phi(z):
    return torch.special.erfc(-z / math.sqrt(2.0)) / 2


def _act(name, z):
    inner = math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
    return {"NONE": z, "RELU": z.clamp(min=0), "GELU": z * _phi(z), "GELU_TANH": z * (1 + torch.tanh(inner)) / 2, "SILU": z * torch.sigmoid(z)}[name]


def _act_grad(name, z):
    z = z.clone().requires_grad_(True)
    with torch.enable_grad():
        return torch.autograd.grad(_act(name, z).sum(), z)[0]


def _make(shape, std, dtype, gen, pad=0):
    """On the GPU, rows `pad` elements apart; what lies between them is NaN."""
    rows, cols = shape
    x = torch.full((rows, cols + pad), float("nan"), dtype=dtype)
    x[:, :cols] = (torch.randn(rows, cols, generator=gen) * std).to(dtype)
    return x.cuda()[:, :cols]


def _flat(shapes, std, dtype, gen, shift):
    """Parameters side by side in a flat array after `shift` others."""
    total = shift + sum(math.prod(s) for s in shapes)
    flat = (torch.randn(total, generator=gen) * std).to(dtype).cuda()
    out, at = [], shift
    for s in shapes:
        out.append(flat[at:at + math.prod(s)].view(s))
        at += math.prod(s)
    return out


def _close(got, want, bound, what):
    got, want = got.double().cpu(), want.cpu()
    assert got.shape == want.shape
    err = (got - want).abs()
    worst = float((err / bound.cpu()).max()) if err.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.3g} of the bound"


def _sum_bound(L, squares):
    """Accumulation in fp32 of L products whose squares sum to `squares`."""
    return 8 * 2.0 ** -24 * math.sqrt(L) * squares.sqrt() + 1e-30


def _forward_case(am, dtype, R, M, K, N, act, bias, residual, pre, pad=0, shift=0, seed=0):
    print("linear", dtype, R, M, K, N, act, bias, residual, pre, pad, shift, flush=True)
    gen = torch.Generator().manual_seed(seed)
    x = [_make((M, K), 1.0, dtype, gen, pad) for _ in range(R)]
    wb = [_flat([(N,), (N, K)], 1 / math.sqrt(K), dtype, gen, shift) for _ in range(R)]
    b, w = [p[0] for p in wb], [p[1] for p in wb]
    r = [_make((M, N), 1.0, dtype, gen, pad) for _ in range(R)] if residual else None
    out = am.linear(x, w, b if bias else None, act=getattr(am, "ACT_" + act), residual=r, with_pre=pre)
    ys, zs = out if pre else (out, None)
    for i in range(R):
        X, W = x[i].double(), w[i].double()
        z = X @ W.t()
        slack = _sum_bound(K, (X * X) @ (W * W).t())
        if bias:
            z = z + b[i].double()
            slack = slack + 2.0 ** -23 * z.abs()
        y = _act(act, z)
        # act is at most 1.13 steep, and rounds like fp32 itself
        slack = 1.2 * slack + 2.0 ** -20 * z.abs().clamp(min=1.0) * (act != "NONE")
        if residual:
            y = y + r[i].double()
            slack = slack + 2.0 ** -23 * y.abs()
        _close(ys[i], y, slack + UNIT[dtype] * (y.abs() + slack) + 1e-30, f"y[{i}]")
        if pre:
            _close(zs[i], z, slack + UNIT[dtype] * (z.abs() + slack) + 1e-30, f"pre[{i}]")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,K,N", [(1, 1, 1), (1, 64, 16), (3, 7, 5), (16, 768, 768), (17, 129, 257), (64, 64, 64), (65, 65, 63), (255, 200, 136),
                                   (300, 31, 1000), (129, 2049, 40), (513, 72, 520)])
def test_products_of_every_shape(amlib, dtype, M, K, N):
    _forward_case(amlib, dtype, 2, M, K, N, "NONE", True, False, False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("residual,pre", [(False, True), (True, False), (True, True)])
def test_epilogue(amlib, dtype, act, residual, pre):
    _forward_case(amlib, dtype, 1, 70, 96, 150, act, True, residual, pre, seed=1)
    _forward_case(amlib, dtype, 3, 33, 1500, 75, act, False, residual, pre, pad=3, shift=1, seed=2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (8, 8), (5, 3)])
def test_places_in_a_flat_array_and_row_strides(amlib, dtype, pad, shift):
    _forward_case(amlib, dtype, 2, 140, 136, 264, "SILU", True, True, True, pad=pad, shift=shift, seed=3)


@pytest.mark.parametrize("R,M,K,N", [(4, 512, 512, 2048), (2, 1111, 1152, 2307), (32, 64, 256, 64), (1, 2048, 2048, 768), (1, 4, 8192, 72)])
def test_larger_products(amlib, R, M, K, N):
    _forward_case(amlib, torch.bfloat16, R, M, K, N, "GELU_TANH", True, True, True, seed=4)


@pytest.mark.parametrize("M,K,N,shift", [(700, 1500, 1300, 1), (600, 1001, 1024, 0), (1024, 1204, 640, 1), (640, 1100, 2050, 3)])
def test_operands_that_are_moved_to_aligned_rows_first(amlib, M, K, N, shift):
    for dtype in (torch.bfloat16, torch.float32):
        _forward_case(amlib, dtype, 2, M, K, N, "SILU", True, False, True, shift=shift, seed=6)
        _backward_case(amlib, dtype, dtype, 2, M, K, N, "NONE", shift=shift, seed=7)
        _backward_case(amlib, dtype, torch.float32, 1, M, K, N, "RELU", pad=1, shift=shift, seed=8)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 8, 9])
def test_few_rows(amlib, dtype, M):
    """Where every weight is read once for all rows, at widths that are no multiples of what a workgroup takes."""
    _forward_case(amlib, dtype, 2, M, 4097, 261, "GELU", True, True, True, pad=1, shift=3, seed=9)
    _forward_case(amlib, dtype, 1, M, 2048, 1024, "NONE", False, False, False, seed=10)
    _forward_case(amlib, dtype, 3, M, 5, 3, "SILU", True, False, True, seed=11)


def _backward_case(am, dtype, grad_dtype, R, M, K, N, act, bias=True, accumulate=False, need_dx=True, need_dw=True, pad=0, shift=0, seed=0):
    print("linear_backward", dtype, grad_dtype, R, M, K, N, act, bias, accumulate, need_dx, need_dw, pad, shift, flush=True)
    gen = torch.Generator().manual_seed(seed)
    x = [_make((M, K), 1.0, dtype, gen, pad) for _ in range(R)]
    dy = [_make((M, N), 1.0, dtype, gen, pad) for _ in range(R)]
    z = [_make((M, N), 1.5, dtype, gen, pad) for _ in range(R)] if act != "NONE" else None
    w = [_flat([(N, K)], 1.0, dtype, gen, shift)[0] for _ in range(R)]
    grads = [_flat([(N,), (N, K), (7,)], 1.0, grad_dtype, gen, shift) for _ in range(R)]
    before = [[g.clone() for g in gs] for gs in grads]
    dx = am.linear_backward(dy, x, w, act=getattr(am, "ACT_" + act), pre=z, dw=[g[1] for g in grads] if need_dw else None,
                            db=[g[0] for g in grads] if bias else None, accumulate=accumulate, need_dx=need_dx)
    assert (dx is None) == (not need_dx)
    for i in range(R):
        X, W, DZ = x[i].double(), w[i].double(), dy[i].double()
        rounded = 0.0
        if act != "NONE":
            DZ = DZ * _act_grad(act, z[i].double())
            rounded = UNIT[dtype] + 2.0 ** -18           # dz as the products see it, and act' itself
        if need_dx:
            want, sq = DZ @ W, (DZ * DZ) @ (W * W)
            slack = _sum_bound(N, sq) + 5 * rounded * sq.sqrt() + 2.0 ** -18 * W.abs().sum(0) * (act != "NONE")
            _close(dx[i], want, slack + UNIT[dtype] * (want.abs() + slack) + 1e-30, f"dx[{i}]")
        for name, wanted, g, old, want, sq, L in (
                ("dw", need_dw, grads[i][1], before[i][1], DZ.t() @ X, (DZ * DZ).t() @ (X * X), M),
                ("db", bias, grads[i][0], before[i][0], DZ.sum(0), (DZ * DZ).sum(0), M)):
            if not wanted:
                assert torch.equal(g, old)
                continue
            slack = _sum_bound(max(L, 1), sq) + (5 * rounded * sq.sqrt() if name == "dw" else 2.0 ** -18 * math.sqrt(M) * (act != "NONE"))
            if act != "NONE" and name == "dw":
                slack = slack + 2.0 ** -18 * X.abs().sum(0)
            if accumulate:
                want = want + old.double()
                slack = slack + 2.0 ** -23 * want.abs()
            _close(g, want, slack + UNIT[grad_dtype] * (want.abs() + slack) + 1e-30, f"{name}[{i}]")
        assert torch.equal(grads[i][2], before[i][2])            # what lies after them is left alone


TYPES = [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32)]


@pytest.mark.parametrize("dtype,grad_dtype", TYPES)
@pytest.mark.parametrize("M,K,N", [(1, 1, 1), (1, 40, 24), (3, 5, 7), (64, 64, 64), (67, 129, 65), (200, 136, 255), (33, 1000, 31), (1025, 40, 72),
                                   (520, 513, 72)])
def test_gradients_of_every_shape(amlib, dtype, grad_dtype, M, K, N):
    _backward_case(amlib, dtype, grad_dtype, 2, M, K, N, "NONE")


@pytest.mark.parametrize("dtype,grad_dtype", TYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradients_of_activations(amlib, dtype, grad_dtype, act, accumulate):
    _backward_case(amlib, dtype, grad_dtype, 2, 77, 96, 150, act, accumulate=accumulate, pad=3, shift=1, seed=1)


@pytest.mark.parametrize("bias,need_dx,need_dw", [(True, False, False), (False, True, False), (False, False, True), (True, True, False)])
@pytest.mark.parametrize("act", ["NONE", "SILU"])
def test_gradients_one_by_one(amlib, act, bias, need_dx, need_dw):
    _backward_case(amlib, torch.bfloat16, torch.float32, 2, 90, 72, 130, act, bias=bias, need_dx=need_dx, need_dw=need_dw, seed=2)


@pytest.mark.parametrize("R,M,K,N,act", [(4, 512, 2048, 512, "NONE"), (3, 1111, 1152, 2307, "GELU_TANH"), (1, 4096, 256, 256, "NONE"), (8, 256, 320, 320, "GELU")])
def test_larger_gradients(amlib, R, M, K, N, act):
    _backward_case(amlib, torch.bfloat16, torch.bfloat16, R, M, K, N, act, seed=3)


@pytest.mark.parametrize("act", ACTS[1:])
def test_gradients_against_differences(amlib, act):
    """dx, dw and db of fp32 inputs against central differences of the forward call itself: step h = 2^-6, error h^2/6 |f'''| (below
    2^-13 times the row's terms) plus the rounding of two sums over 2h."""
    am = amlib
    gen = torch.Generator().manual_seed(5)
    M, K, N, h = 5, 12, 9, 2.0 ** -6
    x, w = torch.randn(M, K, generator=gen).cuda(), (torch.randn(N, K, generator=gen) / 4).cuda()
    b, dy = torch.randn(N, generator=gen).cuda(), torch.randn(M, N, generator=gen).cuda()
    code = getattr(am, "ACT_" + act)
    _, pre = am.linear([x], [w], [b], act=code, with_pre=True)
    if act == "RELU":                      # no difference across the kink
        assert float(pre[0].abs().min()) > 1e-4
        h = 2.0 ** -15
    dw, db = torch.zeros_like(w), torch.zeros_like(b)
    dx = am.linear_backward([dy], [x], [w], act=code, pre=pre, dw=[dw], db=[db])[0]

    def value():
        return float((am.linear([x], [w], [b], act=code)[0].double() * dy.double()).sum())

    for t, grad in ((x, dx), (w, dw), (b, db)):
        flat, g = t.view(-1), grad.reshape(-1).cpu()
        for j in range(0, flat.numel(), max(1, flat.numel() // 16)):
            keep = float(flat[j])
            flat[j] = keep + h
            up = value()
            step = float(flat[j])
            flat[j] = keep - h
            down = value()
            step -= float(flat[j])
            flat[j] = keep
            slope = (up - down) / step
            assert abs(slope - float(g[j])) <= 2.0 ** -11 * 20 + 2.0 ** -24 * 200 / h, (act, j, slope, float(g[j]))


def test_no_rows(amlib):
    am = amlib
    x, w, b = torch.empty(0, 12, device="cuda"), torch.ones(5, 12, device="cuda"), torch.ones(5, device="cuda")
    y, pre = am.linear([x], [w], [b], act=am.ACT_GELU, with_pre=True)
    assert y[0].shape == (0, 5) and pre[0].shape == (0, 5)
    dw, db = torch.ones(5, 12, device="cuda"), torch.ones(5, device="cuda")
    dy = torch.empty(0, 5, device="cuda")
    assert am.linear_backward([dy], [x], [w], dw=[dw], db=[db], accumulate=True)[0].shape == (0, 12)
    assert bool((dw == 1).all()) and bool((db == 1).all())
    am.linear_backward([dy], [x], [w], act=am.ACT_SILU, pre=[dy], dw=[dw], db=[db])
    assert not dw.any() and not db.any()


def test_values_that_are_not_finite_stay_where_they_belong(amlib):
    """A NaN row of x reaches its own row of y alone; an infinite weight its own column."""
    am = amlib
    for dtype in (torch.bfloat16, torch.float32):
        x, w = torch.ones(70, 72, dtype=dtype, device="cuda"), torch.ones(80, 72, dtype=dtype, device="cuda")
        x[69, 71] = float("nan")
        w[79, 3] = float("inf")
        y = am.linear([x], [w])[0]
        assert bool(y[69].isnan().all()) and not bool(y[:69].isnan().any())
        assert bool(y[:69, 79].isinf().all()) and bool((y[:69, :79] == 72).all())


def test_same_result_on_another_stream_and_again(amlib):
    am = amlib
    gen = torch.Generator().manual_seed(7)
    x, w = [_make((300, 4096), 1.0, torch.bfloat16, gen)], [_make((96, 4096), 1.0, torch.bfloat16, gen)]
    first = am.linear(x, w)[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = am.linear(x, w)[0]
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first, again)


def test_in_a_graph(amlib):
    am = amlib
    gen = torch.Generator().manual_seed(8)
    x, w = [_make((64, 2048), 1.0, torch.bfloat16, gen)], [_make((128, 2048), 1.0, torch.bfloat16, gen)]
    dy, dw = [_make((64, 128), 1.0, torch.bfloat16, gen)], [torch.empty(128, 2048, device="cuda")]
    am.linear(x, w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = am.linear(x, w, act=am.ACT_RELU)
        dx = am.linear_backward(dy, x, w, dw=dw)
    for k in range(3):
        x[0].copy_(_make((64, 2048), 1.0, torch.bfloat16, gen))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y[0], dx[0], dw[0])]
        want = [am.linear(x, w, act=am.ACT_RELU)[0], am.linear_backward(dy, x, w, dw=dw)[0], dw[0]]
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k
