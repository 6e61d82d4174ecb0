"""What the layers' Python entry points refuse, with tensors on the GPU; nothing is launched."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def _t(*shape, dtype=BF):
    return torch.zeros(shape, dtype=dtype, device="cuda")


@pytest.mark.parametrize("kw", [
    dict(x=[_t]), dict(w=[_t]),
], ids=["x", "w"])
def test_not_tensors(amlib, kw):
    args = dict(x=[_t(4, 8)], w=[_t(3, 8)])
    args.update(kw)
    with pytest.raises(ValueError):
        amlib.linear(**args)


def test_linear(amlib):
    am, x, w = amlib, _t(4, 8), _t(3, 8)
    bad = [dict(x=[x, x]), dict(x=[_t(4, 9)]), dict(w=[_t(3, 8, dtype=torch.float32)]), dict(x=[_t(8)]), dict(x=[_t(8, 4).t()]), dict(x=[_t(1, 8).expand(4, 8)]),
           dict(w=[_t(3, 16)[:, ::2]]), dict(w=[_t(3, 9)[:, :8]]), dict(bias=[_t(4)]), dict(bias=[_t(3, dtype=torch.float32)]), dict(residual=[_t(4, 4)]),
           dict(x=[_t(4, 8).half()], w=[_t(3, 8).half()]), dict(x=[_t(4, 8).cpu()]), dict(w=[_t(0, 8)]), dict(x=[_t(4, 0)], w=[_t(3, 0)]),
           dict(x=[x, _t(4, 16)[:, :8]], w=[w, w])]
    for kw in bad:
        args = dict(x=[x], w=[w])
        args.update(kw)
        with pytest.raises(ValueError):
            am.linear(**args)
    with pytest.raises(am.AsyncMeshError):
        am.linear([x], [w], act=9)


def test_linear_backward(amlib):
    am = amlib
    good = dict(dy=[_t(4, 3)], x=[_t(4, 8)], w=[_t(3, 8)])
    for kw in (dict(dy=[_t(4, 4)]), dict(need_dx=False), dict(act=am.ACT_SILU), dict(act=am.ACT_SILU, pre=[_t(4, 4)]), dict(dw=[_t(3, 8, dtype=torch.float16)]),
               dict(dw=[_t(3, 16)[:, :8]]), dict(dw=[_t(3, 8, dtype=torch.float32)], db=[_t(3)]), dict(db=[_t(4)]), dict(dw=[None])):
        with pytest.raises(ValueError):
            am.linear_backward(**{**good, **kw})


def test_qk_norm(amlib):
    am = amlib
    cos, sin = am.rotation_table(5, 16)
    good = dict(q=[_t(5, 2, 16)], k=[_t(5, 1, 16)], q_gain=[_t(16)], k_gain=[_t(16)], cos=cos, sin=sin)
    am.qk_norm(**good)
    for kw in (dict(q=[_t(5, 32)]), dict(k=[_t(4, 1, 16)]), dict(k=[_t(5, 1, 8)]), dict(q=[_t(5, 16, 2).transpose(1, 2)]), dict(q=[_t(5, 4, 16)[:, ::2]]),
               dict(q_gain=[_t(8)]), dict(cos=cos.double()), dict(cos=cos[:, :4]), dict(positions=[torch.zeros(5, dtype=torch.int64, device="cuda")]),
               dict(positions=[torch.zeros(4, dtype=torch.int32, device="cuda")]), dict(q=[_t(1, 2, 16).expand(5, 2, 16)])):
        with pytest.raises(ValueError):
            am.qk_norm(**{**good, **kw})
    with pytest.raises(am.AsyncMeshError):
        am.qk_norm(**good, eps=0.0)
    for kw in (dict(dq=[_t(5, 4, 16)[:, ::2]]), dict(dq=[_t(5, 1, 16)]), dict(dq_gain=[_t(8)]), dict(dq_gain=[_t(16).half()]),
               dict(dq_gain=[_t(16)], dk_gain=[_t(16, dtype=torch.float32)])):
        with pytest.raises(ValueError):
            am.qk_norm_backward(**{**dict(dq=[_t(5, 2, 16)], dk=[_t(5, 1, 16)], **good), **kw})


def test_gradient_norm(amlib):
    am, a, b = amlib, _t(5), _t(7, 2)
    for grads, kw in (([[a, b], [a]], {}), ([[a], [b]], {}), ([[a, b.t()]], {}), ([[a.half()]], {}), ([[a.cpu()]], {}), ([[a, a.cpu()]], {}), ([[None]], {}), ([], {}),
                      ([[a, b]], dict(out=[_t(18)])), ([[a, b]], dict(out=[_t(19).half()])), ([[a, b]], dict(out=[_t(38)[::2]])), ([[a], [a]], dict(out=[_t(5)])),
                      ([[a], [_t(5, dtype=torch.float32)]], {}), ([[a], [a]], dict(out=[_t(5), _t(5, dtype=torch.float32)]))):
        with pytest.raises(ValueError):
            am.grad_norm(grads, **kw)
    with pytest.raises(am.AsyncMeshError):
        am.grad_norm([[a]], max_norm=-1.0)
