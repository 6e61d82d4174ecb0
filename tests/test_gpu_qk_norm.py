"""am_qk_norm and am_qk_norm_backward against the same formulas in 64 bits.

Bounds, in units of fp32 (2^-24) of the values' sizes: the mean square of D <= 512 numbers sums lanes and a butterfly (at most 16 in a
row, all positive), the root, two products, the rotation: below 24 units of the pair's length; an output is rounded once more (2^-8 of
itself in bf16).  Backward: the dot product over D terms adds 24 units of |n| mean |dn n|.  A gain's gradient sums tokens x heads
terms in fp32 runs of at most `run` and joins them in fp64: run units of the sum of their magnitudes at worst; sqrt of it times eight, as
roundings are as often up as down."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
OUT = {BF: 2.0 ** -8, F: 2.0 ** -24}
E = 24 * 2.0 ** -24
EPS = 1e-6


def _inputs(R, T, Hq, Hk, D, dtype, seed, gap=0, shift=0):
    """q and k side by side in the rows of one product, `gap` elements of something else behind, everything `shift` elements into an allocation."""
    gen = torch.Generator().manual_seed(seed)
    width = (Hq + Hk) * D + gap
    qs, ks = [], []
    for _ in range(R):
        flat = (torch.randn(shift + T * width, generator=gen) * 1.3).to(dtype).cuda()
        rows = flat[shift:].view(T, width)
        qs.append(rows[:, :Hq * D].unflatten(1, (Hq, D)) if Hq else torch.empty(T, 0, D, dtype=dtype, device="cuda"))
        ks.append(rows[:, Hq * D:(Hq + Hk) * D].unflatten(1, (Hk, D)) if Hk else torch.empty(T, 0, D, dtype=dtype, device="cuda"))
    gains = [[(1 + 0.2 * torch.randn(D + 1, generator=gen)).to(dtype).cuda()[1:] for _ in range(R)] for _ in range(2)]
    return qs, ks, gains[0], gains[1], gen


def _turn(u, c, s, rot, inter, back=False):
    if back:
        s = -s
    a, b = (u[..., 0:rot:2], u[..., 1:rot:2]) if inter else (u[..., :rot // 2], u[..., rot // 2:rot])
    x, y = a * c - b * s, b * c + a * s
    out = u.clone()
    if inter:
        out[..., 0:rot:2], out[..., 1:rot:2] = x, y
    else:
        out[..., :rot // 2], out[..., rot // 2:rot] = x, y
    return out


def _size(u, rot, inter):
    """The length of every element's pair."""
    v = u.abs()
    if rot:
        a, b = (v[..., 0:rot:2], v[..., 1:rot:2]) if inter else (v[..., :rot // 2], v[..., rot // 2:rot])
        both = a + b
        v = v.clone()
        if inter:
            v[..., 0:rot:2] = v[..., 1:rot:2] = both
        else:
            v[..., :rot // 2] = v[..., rot // 2:rot] = both
    return v


def _rows(positions, T, rows, i):
    return positions[i].long() if positions is not None else torch.arange(T, device="cuda") % max(rows, 1)


def _ok(got, want, bound, what):
    err = (got.double() - want).abs()
    assert got.shape == want.shape
    worst = float((err / bound).max()) if err.numel() else 0.0
    assert worst <= 1, f"{what}: {worst:.3g} of the bound"


def _case(am, R, T, Hq, Hk, D, rot, dtype, inter=False, rows=None, documents=False, gap=0, shift=0, seed=0, grad_dtype=None, accumulate=False):
    print("qk_norm", R, T, Hq, Hk, D, rot, dtype, inter, rows, documents, gap, shift, grad_dtype, accumulate, flush=True)
    q, k, gq, gk, gen = _inputs(R, T, Hq, Hk, D, dtype, seed, gap, shift)
    rows = rows or max(T, 1)
    cos, sin = am.rotation_table(rows, rot)
    positions = [torch.randint(0, rows, (T,), generator=gen).int().cuda() for _ in range(R)] if documents else None
    args = (q, k, gq, gk, cos, sin)
    out = am.qk_norm(*args, positions=positions, eps=EPS, interleaved=inter)
    grad_dtype = grad_dtype or dtype
    d = [[torch.randn(T, H, D, generator=gen).to(dtype).cuda() for _ in range(R)] for H in (Hq, Hk)]
    dg = [[torch.randn(D + 2, generator=gen).to(grad_dtype).cuda() for _ in range(R)] if H else None for H in (Hq, Hk)]
    old = [None if g is None else [x.clone() for x in g] for g in dg]
    dx = am.qk_norm_backward(d[0], d[1], *args, positions=positions, eps=EPS, interleaved=inter, dq_gain=dg[0] and [g[1:-1] for g in dg[0]],
                             dk_gain=dg[1] and [g[1:-1] for g in dg[1]], accumulate=accumulate)
    run = max(256, T)
    for w, (xs, gains, H) in enumerate(((q, gq, Hq), (k, gk, Hk))):
        for i in range(R):
            at = _rows(positions, T, rows, i)
            c, s = cos.double()[at][:, None], sin.double()[at][:, None]
            x, g = xs[i].double(), gains[i].double()
            r = 1 / (x.pow(2).mean(-1, keepdim=True) + EPS).sqrt() if D else x
            n = x * r
            want = _turn(n * g, c, s, rot, inter)
            size = _size(n * g, rot, inter)
            _ok(out[w][i], want, E * size + OUT[dtype] * (want.abs() + E * size) + 1e-30, f"out {w} {i}")
            du = _turn(d[w][i].double(), c, s, rot, inter, back=True)
            dn, dsize = du * g, _size(d[w][i].double(), rot, inter)
            mean = (dn * n).mean(-1, keepdim=True)
            want = r * (dn - n * mean)
            size = r * (dsize * g.abs() + 2 * n.abs() * (dsize * g.abs() * n.abs()).mean(-1, keepdim=True))
            _ok(dx[w][i], want, E * size + OUT[dtype] * (want.abs() + E * size) + 1e-30, f"dx {w} {i}")
            if not H:
                continue
            want, size = (du * n).sum((0, 1)), (dsize * n.abs()).sum((0, 1))
            slack = (E + 8 * math.sqrt(run) * 2.0 ** -24) * size
            if accumulate:
                want = want + old[w][i][1:-1].double()
            _ok(dg[w][i][1:-1], want, slack + OUT[grad_dtype] * (want.abs() + slack) + 1e-30, f"dgain {w} {i}")
            assert torch.equal(dg[w][i][[0, -1]], old[w][i][[0, -1]])


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("D,rot", [(2, 2), (2, 0), (6, 4), (16, 16), (30, 10), (32, 32), (48, 16), (64, 64), (64, 32), (80, 80), (96, 96), (112, 96), (128, 128),
                                   (128, 0), (130, 66), (256, 256), (256, 128), (384, 384), (510, 510), (512, 512)])
@pytest.mark.parametrize("inter", [False, True])
def test_head_sizes_and_rotated_parts(amlib, dtype, D, rot, inter):
    _case(amlib, 2, 9, 3, 2, D, rot, dtype, inter=inter, seed=D)


@pytest.mark.parametrize("T", [1, 2, 63, 1025])
@pytest.mark.parametrize("Hq,Hk", [(1, 1), (12, 12), (8, 1), (0, 3), (5, 0)])
def test_tokens_and_heads(amlib, T, Hq, Hk):
    _case(amlib, 1, T, Hq, Hk, 64, 64, BF, seed=T)
    _case(amlib, 3, T, Hq, Hk, 20, 12, F, inter=True, documents=True, rows=17, seed=T)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("gap,shift", [(0, 0), (64, 0), (7, 0), (64, 1), (3, 3)])
@pytest.mark.parametrize("documents,rows", [(False, 50), (True, 300)])
def test_views_into_a_product_and_positions(amlib, dtype, gap, shift, documents, rows):
    _case(amlib, 2, 120, 4, 2, 96, 96, dtype, rows=rows, documents=documents, gap=gap, shift=shift, seed=5)


@pytest.mark.parametrize("dtype,grad_dtype", [(BF, BF), (BF, F), (F, F)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gains_gradients(amlib, dtype, grad_dtype, accumulate):
    _case(amlib, 2, 300, 6, 3, 64, 32, dtype, grad_dtype=grad_dtype, accumulate=accumulate, seed=6)


def test_many_tokens(amlib):
    _case(amlib, 2, 5000, 16, 4, 128, 128, BF, rows=1024, seed=7)
    _case(amlib, 32, 40, 2, 2, 64, 64, BF, seed=8)


def test_gradients_against_differences(amlib):
    """Central differences of the forward call in fp32: h = 2^-6, error h^2 / 6 |f'''| below 2^-9 of the row's terms, plus rounding over 2 h."""
    am, h = amlib, 2.0 ** -6
    q, k, gq, gk, gen = _inputs(1, 3, 2, 1, 10, F, 9)
    q, k = [q[0].contiguous()], [k[0].contiguous()]
    gq, gk = [gq[0].clone()], [gk[0].clone()]
    cos, sin = am.rotation_table(3, 6)
    d = [torch.randn(3, H, 10, generator=gen).cuda() for H in (2, 1)]
    dgq, dgk = [torch.empty(10, device="cuda")], [torch.empty(10, device="cuda")]
    dq, dk = am.qk_norm_backward([d[0]], [d[1]], q, k, gq, gk, cos, sin, eps=EPS, dq_gain=dgq, dk_gain=dgk)

    def value():
        a, b = am.qk_norm(q, k, gq, gk, cos, sin, eps=EPS)
        return float((a[0].double() * d[0].double()).sum() + (b[0].double() * d[1].double()).sum())

    for t, g in ((q[0], dq[0]), (k[0], dk[0]), (gq[0], dgq[0]), (gk[0], dgk[0])):
        flat, g = t.view(-1), g.reshape(-1).cpu()
        for j in range(0, flat.numel(), max(1, flat.numel() // 12)):
            keep = float(flat[j])
            flat[j] = keep + h
            up, step = value(), float(flat[j])
            flat[j] = keep - h
            down = value()
            step -= float(flat[j])
            flat[j] = keep
            assert abs((up - down) / step - float(g[j])) <= 2.0 ** -9 * 10 + 2.0 ** -24 * 100 / h


def test_a_row_that_the_tables_do_not_have(amlib):
    am = amlib
    q, k, gq, gk, _ = _inputs(1, 4, 1, 1, 32, F, 10)
    cos, sin = am.rotation_table(8, 16)
    positions = [torch.tensor([0, 8, -1, 7], dtype=torch.int32, device="cuda")]
    a, _ = am.qk_norm(q, k, gq, gk, cos, sin, positions=positions)
    assert bool(a[0][[1, 2], :, :16].isnan().all()) and not bool(a[0][[0, 3]].isnan().any()) and not bool(a[0][..., 16:].isnan().any())


def test_zero_rows_and_values_that_are_not_finite(amlib):
    """A head of zeros is divided by sqrt(eps) and stays zero; NaN and infinity stay in their head."""
    am = amlib
    for dtype in (BF, F):
        q, k, gq, gk, _ = _inputs(1, 5, 2, 1, 64, dtype, 11)
        q = [q[0].contiguous()]
        q[0][1, 0] = 0
        q[0][2, 1, 5] = float("nan")
        q[0][3, 0, 6] = float("inf")
        cos, sin = am.rotation_table(5, 64)
        a, _ = am.qk_norm(q, k, gq, gk, cos, sin)
        assert not a[0][1, 0].any() and bool(a[0][2, 1].isnan().all()) and bool(a[0][3, 0].isnan().any())
        rest = torch.ones(5, 2, dtype=torch.bool)
        rest[2, 1] = rest[3, 0] = False
        assert bool(a[0].cpu()[rest].isfinite().all())


def test_no_tokens(amlib):
    am = amlib
    q, k, gq, gk, _ = _inputs(2, 0, 2, 1, 16, F, 12)
    cos, sin = am.rotation_table(4, 16)
    a, b = am.qk_norm(q, k, gq, gk, cos, sin)
    assert a[0].shape == (0, 2, 16) and b[1].shape == (0, 1, 16)
    dg = [torch.ones(16, device="cuda") for _ in range(2)]
    am.qk_norm_backward(a, b, q, k, gq, gk, cos, sin, dq_gain=dg, accumulate=True)
    assert all(bool((g == 1).all()) for g in dg)
    am.qk_norm_backward(a, b, q, k, gq, gk, cos, sin, dq_gain=dg)
    assert not any(bool(g.any()) for g in dg)


def test_in_a_graph(amlib):
    am = amlib
    q, k, gq, gk, gen = _inputs(2, 100, 4, 4, 64, BF, 13)
    cos, sin = am.rotation_table(100, 64)
    d = [torch.randn(100, 4, 64, generator=gen).to(BF).cuda() for _ in range(2)]
    dg = [torch.empty(64, device="cuda") for _ in range(2)]

    def both():
        a, b = am.qk_norm(q, k, gq, gk, cos, sin)
        c, e = am.qk_norm_backward(d, d, q, k, gq, gk, cos, sin, dq_gain=dg)
        return [*a, *b, *c, *e, *dg]

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = both()
    for n in range(3):
        q[0].copy_(torch.randn(100, 4, 64, generator=gen).to(BF))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in kept]
        assert all(torch.equal(x, y) for x, y in zip(got, both())), n
