"""Arrays of more than 2^31 elements: the last rows of a long call against the same rows alone, bit for bit where the sums are the same."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def _fill(n, seed):
    """n values by cycling a drawn million: quick, and no two neighbouring rows alike."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    pool = torch.randn(1_000_003, generator=g, device="cuda").to(BF)
    out = torch.empty(n, dtype=BF, device="cuda")
    at = 0
    while at < n:
        k = min(pool.numel(), n - at)
        out[at:at + k] = pool[:k]
        at += k
    return out


def test_products_of_many_rows(amlib):
    am = amlib
    M, K, N = (1 << 21) + 77, 1032, 64
    print("far offsets: linear", M, K, N, flush=True)
    x, w, b = _fill(M * K, 1).view(M, K), _fill(N * K, 2).view(N, K), _fill(N, 3)
    y = am.linear([x], [w], [b], act=am.ACT_SILU)[0]
    for rows in (slice(0, 256), slice(M - 300, M)):
        part = x[rows].float() @ w.float().t() + b.float()
        want = part * torch.sigmoid(part)
        assert bool(((y[rows].float() - want).abs() <= 2.0 ** -7 * want.abs() + 2.0 ** -10).all())
    # the gradient of x (that of w sums all rows; its own test is in small sizes) and the column sums
    dy = _fill(M * N, 4).view(M, N)
    db = torch.empty(N, device="cuda")
    dx = am.linear_backward([dy], [x], [w], db=[db])[0]
    for rows in (slice(0, 256), slice(M - 300, M)):
        want = dy[rows].float() @ w.float()
        assert bool(((dx[rows].float() - want).abs() <= 2.0 ** -7 * want.abs() + 2.0 ** -8).all())
    want = dy.sum(0, dtype=torch.float64)
    assert bool(((db.double() - want).abs() <= 2.0 ** -20 * dy.abs().sum(0, dtype=torch.float64)).all())


def test_heads_of_many_tokens(amlib):
    am = amlib
    T, H, D = 270_001, 64, 128
    print("far offsets: qk_norm", T, H, D, flush=True)
    q = _fill(T * H * D, 5).view(T, H, D)
    k, gain = torch.zeros(T, 0, D, dtype=BF, device="cuda"), _fill(D, 6)
    cos, sin = am.rotation_table(1000, D)
    out = am.qk_norm([q], [k], [gain], [gain], cos, sin)[0][0]
    tail = slice(T - 1001, T)
    positions = [(torch.arange(T - 1001, T, device="cuda") % 1000).int()]
    alone = am.qk_norm([q[tail]], [k[tail]], [gain], [gain], cos, sin, positions=positions)[0][0]
    assert torch.equal(out[tail], alone)


def test_the_norm_of_a_long_tensor(amlib):
    n = (1 << 31) + 12_345
    print("far offsets: grad_norm", n, flush=True)
    g = torch.zeros(n, dtype=BF, device="cuda")
    g[-1], g[n // 2], g[0] = 3.0, 4.0, 12.0
    out = torch.ones(n + 1, dtype=BF, device="cuda")
    norm, factor = amlib.grad_norm([[g[:1], g[1:]]], 6.5, out=[out[:n]])
    assert float(norm) == 13.0 and float(factor) == 0.5 and float(out[n]) == 1.0
    assert float(out[n - 1]) == 3.0 and float(out[n // 2]) == 4.0 and int(torch.count_nonzero(out[:n])) == 3
    amlib.clip_grads([[g]], 6.5)
    assert float(g[-1]) == 1.5 and float(g[0]) == 6.0
